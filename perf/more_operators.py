"""Timed cases of what a model with rotary positions or a latent cache asks of the paged 8-bit cache.

  rotate       rotary positions of queries or keys, and the gradient (the turn back)
  kv_store     keys turned and, with the values, written into 8-bit pages; the step's
               queries turned beside them
  latent_store one latent vector and one rotary key a token into 8-bit pages, a
               power-of-two scale for each token and part; queries turned beside them
  latent       absorbed form: every head's query against the same paged latents, which
               are keys and values at once
  expanded     expanded form: a prompt's keys of a head and one rotary key that all
               heads share, values of another width, ragged and causal

Caches: keys and values as in perf/operators.py; latents as codes [pages, page tokens,
latent + rotary], one byte each, with exponent bytes [pages, page tokens, 2]: a value is
code * 2^(exponent byte - 127).
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}
CODES = {"e4m3fn": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
CODE_MAX = {"e4m3fn": 448.0, "e5m2": 57344.0}      # 1.75 * 2^8 and 1.75 * 2^15
CODE_TOP = {"e4m3fn": 8, "e5m2": 15}
EXP_MIN = 27                                        # least exponent byte: scale 2^-100
EXP_MAX = {"e4m3fn": 246, "e5m2": 239}              # the largest scaled code stays finite in 32 bits


def listed():
    return [
        # queries of a long prompt, a slice of the fused projection
        {"name": "rotate_prompt", "op": "rotate", "rows": 16384, "heads": 32, "dim": 128, "rot": 128, "first": 0, "type": "bf16",
         "interleaved": False, "inverse": False, "fused": True, "far": 16384, "magnitude": 1.0},
        # gradient of a training step: the rotary part at the end of odd heads, pairs side by side, far positions, scaled
        {"name": "rotate_grad", "op": "rotate", "rows": 4099, "heads": 11, "dim": 104, "rot": 40, "first": 64, "type": "fp32",
         "interleaved": True, "inverse": True, "fused": False, "far": 1 << 20, "magnitude": 1.2},
        # a decode step of 64 requests: places, then queries, keys and values of a layer in one call
        {"name": "kv_step", "op": "kv_store", "reqs": 64, "ctx_lo": 100, "ctx_hi": 8000, "new_lo": 1, "new_hi": 1, "page": 64, "kv": 8,
         "heads": 32, "dim": 128, "rot": 128, "type": "bf16", "code": "e4m3fn", "interleaved": False, "magnitude": 1.0},
        # prompts enter
        {"name": "kv_prompt", "op": "kv_store", "reqs": 8, "ctx_lo": 0, "ctx_hi": 0, "new_lo": 2048, "new_hi": 2048, "page": 64, "kv": 8,
         "heads": 32, "dim": 128, "rot": 128, "type": "bf16", "code": "e4m3fn", "interleaved": False, "magnitude": 1.0},
        # ragged pieces of a few prompts, pairs side by side
        {"name": "lstore_pieces", "op": "latent_store", "reqs": 37, "ctx_lo": 0, "ctx_hi": 3001, "new_lo": 1, "new_hi": 41, "page": 16,
         "heads": 7, "latent": 256, "rot": 32, "type": "fp16", "code": "e5m2", "interleaved": True, "magnitude": 1.1},
        # a prompt's latents; the queries are turned elsewhere
        {"name": "lstore_prompt", "op": "latent_store", "reqs": 4, "ctx_lo": 0, "ctx_hi": 0, "new_lo": 4096, "new_hi": 4096, "page": 64,
         "heads": 0, "latent": 512, "rot": 64, "type": "bf16", "code": "e4m3fn", "interleaved": False, "magnitude": 1.0},
        # one request that has just begun
        {"name": "latent_one", "op": "latent", "reqs": 1, "ctx_lo": 37, "ctx_hi": 37, "new_lo": 1, "new_hi": 1, "page": 16, "heads": 16,
         "latent": 512, "rot": 64, "type": "bf16", "code": "e4m3fn"},
        # a decode step, few heads on this GPU: bound by the cache's bytes
        {"name": "latent_step", "op": "latent", "reqs": 64, "ctx_lo": 1, "ctx_hi": 8190, "new_lo": 1, "new_hi": 1, "page": 64, "heads": 16,
         "latent": 512, "rot": 64, "type": "bf16", "code": "e4m3fn"},
        # a decode step with all heads on one GPU: bound by products
        {"name": "latent_heads", "op": "latent", "reqs": 32, "ctx_lo": 1000, "ctx_hi": 16383, "new_lo": 1, "new_hi": 1, "page": 64,
         "heads": 128, "latent": 512, "rot": 64, "type": "bf16", "code": "e4m3fn"},
        # pieces of two prompts over what they hold already
        {"name": "latent_chunk", "op": "latent", "reqs": 2, "ctx_lo": 5001, "ctx_hi": 8003, "new_lo": 200, "new_hi": 256, "page": 128,
         "heads": 12, "latent": 256, "rot": 32, "type": "fp16", "code": "e5m2"},
        # a prompt in the expanded form
        {"name": "expanded_prompt", "op": "expanded", "reqs": 1, "ctx_lo": 0, "ctx_hi": 0, "new_lo": 4096, "new_hi": 4096, "heads": 16,
         "nope": 128, "rot": 64, "value": 128, "type": "bf16", "fused": True},
        # ragged prompts, some with keys of earlier pieces
        {"name": "expanded_ragged", "op": "expanded", "reqs": 7, "ctx_lo": 0, "ctx_hi": 900, "new_lo": 1, "new_hi": 1433, "heads": 6,
         "nope": 64, "rot": 32, "value": 64, "type": "fp16", "fused": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["rotate", "kv_store", "latent_store", "latent", "latent", "expanded"])
    while True:
        case = {"op": op, "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
        if op == "rotate":
            dim = rng.choice([64, 80, 96, 128, 192, 256, rng.randrange(16, 257)])
            rot = rng.choice([dim - dim % 2, 2 * rng.randrange(1, dim // 2 + 1), dim // 4 * 2])
            case |= {"rows": _log(rng, 1, 16384), "heads": rng.choice([1, 2, 3, 8, 12, 14, 32, 64]), "dim": dim, "rot": rot,
                     "first": rng.choice([0, dim - rot, rng.randrange(dim - rot + 1)]), "interleaved": rng.random() < 0.5,
                     "inverse": rng.random() < 0.4, "fused": rng.random() < 0.5, "far": _log(rng, 1, 1 << 20),
                     "magnitude": rng.choice([1.0, 1.25])}
            if case["rows"] * case["heads"] * dim * SIZES[case["type"]] <= 16384 * 32 * 128 * 2:
                return case
            continue
        case["reqs"] = _log(rng, 1, 64)
        if op == "expanded":
            case["type"] = rng.choice(["bf16", "bf16", "fp16"])
            case |= {"ctx_lo": 0, "ctx_hi": rng.choice([0, _log(rng, 1, 4096)]), "new_lo": 1, "new_hi": _log(rng, 1, 4096),
                     "heads": rng.choice([1, 2, 3, 8, 16, 24]), "nope": rng.choice([64, 128]), "rot": rng.choice([32, 64]),
                     "value": rng.choice([64, 128]), "fused": rng.random() < 0.5}
            case["new_lo"] = rng.choice([1, case["new_hi"]])
            ctx, new = _lengths(case)
            longest = max(c + n for c, n in zip(ctx, new))
            if len(ctx) * case["heads"] * max(new) * longest <= 1 << 28 and _tokens(case) * case["heads"] * 192 <= 1 << 26:
                return case
            continue
        case |= {"page": rng.choice([16, 32, 64, 128, 256]), "code": rng.choice(["e4m3fn", "e4m3fn", "e5m2"])}
        if op != "latent":
            case |= {"ctx_lo": rng.randrange(64), "ctx_hi": 64 + _log(rng, 1, 8000), "new_lo": 1, "new_hi": rng.choice([1, _log(rng, 1, 8192)]),
                     "interleaved": rng.random() < 0.5, "magnitude": rng.choice([1.0, 1.25])}
            if op == "kv_store":
                kv, dim = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 96, 128, 192, 256])
                case |= {"kv": kv, "heads": rng.choice([0, 1, 4, 7]) * kv, "dim": dim, "rot": rng.choice([dim, dim, dim // 2, 2 * rng.randrange(1, dim // 2)])}
                if _tokens(case) * (2 * kv + case["heads"]) * dim * SIZES[case["type"]] <= 16384 * 48 * 128 * 2:
                    return case
                continue
            case |= {"heads": rng.choice([0, 1, 7, 16]), "latent": rng.choice([256, 512]), "rot": rng.choice([32, 64])}
            if _tokens(case) * (576 + 64 * case["heads"]) <= 16384 * 576 * 2:
                return case
            continue
        case["type"] = rng.choice(["bf16", "bf16", "fp16"])
        case |= {"ctx_lo": rng.randrange(64), "ctx_hi": 64 + _log(rng, 1, 60000), "new_lo": 1, "new_hi": rng.choice([1, 1, rng.randrange(2, 10), _log(rng, 10, 512)]),
                 "heads": rng.choice([1, 2, 3, 8, 12, 16, 32, 64, 128]), "latent": rng.choice([256, 512]), "rot": rng.choice([32, 64])}
        ctx, new = _lengths(case)
        longest = max(c + n for c, n in zip(ctx, new))
        if len(ctx) * case["heads"] * max(new) * longest <= 1 << 26 and len(ctx) * longest * 576 <= 1 << 29:
            return case


# ------------------------------------------------------------------ the case's requests
def _spread(lo, hi, count):
    return [lo + (hi - lo) * i // max(1, count - 1) for i in range(count)]


def _lengths(case):
    """Tokens held and new tokens of each request: the same whatever the seed, which only orders them."""
    n = case["reqs"]
    ctx, new = _spread(case["ctx_lo"], case["ctx_hi"], n), _spread(case["new_lo"], case["new_hi"], n)
    return ctx, [new[(i * 7 + 3) % n] for i in range(n)] if n % 7 else new  # long pieces do not go with long contexts


def _tokens(case):
    return sum(_lengths(case)[1])


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _values(shape, sigma, g):
    return torch.randn(shape, device=DEVICE, generator=g) * sigma


def _sigma(shape, g):
    """Channel scales: log-normal, four channels ten times as large; mean square 1."""
    sigma = torch.exp(0.5 * torch.randn(shape, device=DEVICE, generator=g))
    sigma[..., torch.randperm(shape[-1], device=DEVICE, generator=g)[:4]] *= 10
    return sigma / sigma.square().mean(dim=-1, keepdim=True).sqrt()


def _frequencies(rot):
    return (10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEVICE) / rot)).float()


def prepare(case, seed):
    g = _generator(seed)
    kind = TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "rotate":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        x = _values((rows, heads + (2 if case["fused"] else 0), dim), 1.0, g).to(kind)
        s |= {"x": x[:, :heads], "positions": torch.randint(0, case["far"] + 1, (rows,), device=DEVICE, generator=g, dtype=torch.int32),
              "freq": _frequencies(case["rot"]), "out": torch.empty(rows, heads, dim, dtype=kind, device=DEVICE)}
        return s
    ctx, new = _lengths(case)
    reqs, tokens = len(ctx), _tokens(case)
    order = torch.randperm(reqs, device=DEVICE, generator=g)
    ctx = torch.tensor(ctx, dtype=torch.int64, device=DEVICE)[order]
    new = torch.tensor(new, dtype=torch.int64, device=DEVICE)[order]
    total = ctx + new
    zero = new.new_zeros(1)
    s |= {"tokens": tokens, "lens": total.to(torch.int32), "q_start": torch.cat([zero, torch.cumsum(new, 0)]).to(torch.int32)}
    if case["op"] == "expanded":
        keys, heads, nope, rot, value = int(total.sum()), case["heads"], case["nope"], case["rot"], case["value"]
        kv = _values((keys, heads, nope + value), 1.0, g).to(kind)
        s |= {"q": _values((tokens, heads, nope + rot), 1.5, g).to(kind), "k_rot": _values((keys, rot), 1.0, g).to(kind),
              "k": kv[..., :nope], "v": kv[..., nope:], "k_start": torch.cat([zero, torch.cumsum(total, 0)]).to(torch.int32),
              "max_new": int(new.max()), "max_len": int(total.max()), "scale": (nope + rot) ** -0.5}
        if not case["fused"]:                                             # each in memory of its own
            s |= {"k": s["k"].contiguous(), "v": s["v"].contiguous()}
        s["out"] = torch.empty(tokens, heads, value, dtype=kind, device=DEVICE)
        s["lse"] = torch.empty(tokens, heads, dtype=torch.float32, device=DEVICE)
        return s
    page = case["page"]
    done = case["op"] == "latent"
    max_pages = int(((total + page - 1) // page).max()) + 1
    held = (total + page - 1) // page
    pool = int(held.sum()) + 3                                            # the last page is never handed out
    pages = torch.randperm(pool - 1, device=DEVICE, generator=g).to(torch.int32)
    at = torch.arange(max_pages, device=DEVICE)
    first = torch.cumsum(held, 0) - held
    s["table"] = torch.where(at < held[:, None], pages[(first[:, None] + at).clamp(max=pool - 2)], -1).to(torch.int32).contiguous()
    if not done:
        _places(s, ctx, new, page, g)
        s |= {"freq": _frequencies(case["rot"]), "positions": torch.zeros(tokens, dtype=torch.int32, device=DEVICE)}
    heads, code = case["heads"], case["code"]
    if case["op"] == "kv_store":
        kv, dim = case["kv"], case["dim"]
        sigma_k, sigma_v = _sigma((kv, dim), g), _sigma((kv, dim), g)
        k, s["k_exp"] = _fill(pool, kv, page, dim, sigma_k, code, g)
        v, s["v_exp"] = _fill(pool, kv, page, dim, sigma_v, code, g)
        s |= {"k_cache": k, "v_cache": v.transpose(2, 3).contiguous()}
        qkv = torch.cat([_values((tokens, n, dim), sig, g).to(kind) for n, sig in ((heads, 1.0), (kv, sigma_k), (kv, sigma_v))], dim=1)
        s |= {"q": qkv[:, :heads] if heads else None, "k": qkv[:, heads:heads + kv], "v": qkv[:, heads + kv:]}
        s["q_out"] = torch.empty(tokens, heads, dim, dtype=kind, device=DEVICE) if heads else None
        if own:
            import paper_2604_17172_amd as uz
            s["cache"] = uz.KVCache(s["k_cache"], s["k_exp"], s["v_cache"], s["v_exp"], code)
        return s
    latent, rot = case["latent"], case["rot"]
    sigma = torch.cat([_sigma((latent,), g), _sigma((rot,), g)])
    codes = torch.empty(pool, page, latent + rot, dtype=torch.uint8, device=DEVICE)
    exps = torch.empty(pool, page, 2, dtype=torch.uint8, device=DEVICE)
    step = max(1, (1 << 26) // (page * (latent + rot)))
    for a in range(0, pool, step):
        x = _values((min(step, pool - a), page, latent + rot), sigma, g)
        codes[a:a + step], exps[a:a + step] = _latent_codes(x, latent, code)
    s |= {"codes": codes, "exps": exps}
    if own:
        import paper_2604_17172_amd as uz
        s["cache"] = uz.LatentCache(codes, exps, rot, code)
    if not done:
        s |= {"latent": _values((tokens, latent), sigma[:latent], g).to(kind), "k_rot": _values((tokens, rot), sigma[latent:], g).to(kind)}
        # a query's rotary part is turned from the projection's output to where attention reads it
        s["q"] = _values((tokens, heads, 64 + rot), 1.0, g).to(kind)[..., 64:] if heads else None
        s["q_out"] = torch.zeros(tokens, heads, latent + rot, dtype=kind, device=DEVICE)[..., latent:] if heads else None
        return s
    s |= {"q": _values((tokens, heads, latent + rot), 2.0, g).to(kind), "max_new": int(new.max()), "scale": (latent + rot) ** -0.5,
          "out": torch.empty(tokens, heads, latent, dtype=kind, device=DEVICE), "lse": torch.empty(tokens, heads, dtype=torch.float32, device=DEVICE)}
    if own:
        s["ws"] = uz.latent_attend_workspace(s["q"], s["cache"], reqs, s["max_new"])
    return s


def _places(s, ctx, new, page, g):
    """Slots and runs of the new tokens, as the plan of a step leaves them."""
    i = torch.repeat_interleave(torch.arange(new.numel(), device=DEVICE), new)
    j = torch.arange(s["tokens"], device=DEVICE) - s["q_start"].long()[i]
    p = ctx[i] + j
    s["slots"] = s["table"][i, p // page].long() * page + p % page
    begins = ((j == 0) | (p % page == 0)).nonzero()[:, 0]
    runs = torch.zeros(max(1, min(s["tokens"], s["tokens"] // page + 2 * new.numel())), 2, dtype=torch.int32, device=DEVICE)
    runs[:begins.numel(), 0] = begins.to(torch.int32)
    runs[:begins.numel(), 1] = torch.minimum(page - p[begins] % page, (new[i] - j)[begins]).to(torch.int32)
    s |= {"runs": runs, "counts": torch.tensor([0, begins.numel()], dtype=torch.int32, device=DEVICE)}


def _fill(pages, kv, page, dim, sigma, code, g):
    """A pool of keys as earlier steps left it: codes [pages, kv, page, dim] and exponents [pages, kv]."""
    codes = torch.empty(pages, kv, page, dim, dtype=torch.uint8, device=DEVICE)
    exps = torch.empty(pages, kv, dtype=torch.uint8, device=DEVICE)
    step = max(1, (1 << 27) // (kv * page * dim))
    for a in range(0, pages, step):
        x = _values((min(step, pages - a), kv, page, dim), sigma[:, None, :], g)
        e = _exponent(x.abs().amax(dim=(2, 3)), code)
        exps[a:a + step] = e.to(torch.uint8)
        codes[a:a + step] = _encode(x, e[:, :, None, None], code)
    return codes, exps


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"rotate": _rotate_pass, "kv_store": _kv_store, "latent_store": _latent_store, "latent": _latent, "expanded": _expanded}[op](s)
    import paper_2604_17172_amd as uz
    if op == "rotate":
        return uz.rotate(s["x"], s["positions"], s["freq"], interleaved=case["interleaved"], first=case["first"], magnitude=case["magnitude"],
                         inverse=case["inverse"], out=s["out"])
    if op == "kv_store":
        uz.kv_positions(s["lens"], s["q_start"], s["tokens"], out=s["positions"])
        q = uz.kv_rotate_store(s["cache"], s["k"], s["v"], s["positions"], s["freq"], s["slots"], s["runs"], s["counts"], q=s["q"],
                               interleaved=case["interleaved"], magnitude=case["magnitude"], q_out=s["q_out"])
        return _kv_result(s, q)
    if op == "latent_store":
        uz.kv_positions(s["lens"], s["q_start"], s["tokens"], out=s["positions"])
        q = uz.latent_store(s["cache"], s["latent"], s["k_rot"], s["positions"], s["freq"], s["slots"], q=s["q"],
                            interleaved=case["interleaved"], magnitude=case["magnitude"], q_out=s["q_out"])
        return _latent_result(s, q)
    if op == "latent":
        out, lse = uz.latent_attend(s["q"], s["cache"], s["table"], s["lens"], s["q_start"], s["max_new"], s["scale"], out=s["out"],
                                    lse=s["lse"], ws=s["ws"])
    else:
        out, lse = uz.latent_attend_expanded(s["q"], s["k"], s["k_rot"], s["v"], s["q_start"], s["k_start"], s["max_new"], scale=s["scale"],
                                             out=s["out"], lse=s["lse"])
    return {"out": out, "lse": lse}


def _kv_result(s, q):
    """The cache as the values that its codes stand for, the exponents of their scales, and the queries."""
    kind = CODES[s["case"]["code"]]
    r = {"k": s["k_cache"].view(kind), "v": s["v_cache"].view(kind), "k_exp": s["k_exp"], "v_exp": s["v_exp"]}
    return r if q is None else {**r, "q": q}


def _latent_result(s, q):
    r = {"codes": s["codes"].view(CODES[s["case"]["code"]]), "exps": s["exps"]}
    return r if q is None else {**r, "q": q}


# ------------------------------------------------------------------ plain forms
def _turned(x, positions, freq, interleaved, first, magnitude, inverse=False):
    """Rotary positions in 32 bits, the angles in 64: pairs (i, i + rot / 2) or (2 i, 2 i + 1) of the rotary part."""
    angle = positions.double()[:, None] * freq.double()
    cos = (torch.cos(angle) * magnitude).float()[:, None]
    sin = (torch.sin(angle) * (-magnitude if inverse else magnitude)).float()[:, None]
    half = freq.numel()
    x = x.float()
    part = x[..., first:first + 2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :half], part[..., half:])
    u, w = a * cos - b * sin, a * sin + b * cos
    part = torch.stack([u, w], dim=-1).flatten(-2) if interleaved else torch.cat([u, w], dim=-1)
    return torch.cat([x[..., :first], part, x[..., first + 2 * half:]], dim=-1)


def _rotate_pass(s):
    case = s["case"]
    y = _turned(s["x"], s["positions"], s["freq"], case["interleaved"], case["first"], case["magnitude"], case["inverse"])
    return y.to(TYPES[case["type"]])


def _positions(s):
    """The place of each row in its request."""
    row = torch.arange(s["tokens"], device=DEVICE)
    end = s["q_start"][1:].long()
    i = torch.searchsorted(end, row, right=True)
    return s["lens"].long()[i] - end[i] + row


def _power(e):
    """2^(e - 127) in 32 bits, from its exponent byte."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _exponent(amax, code):
    """The least exponent byte whose scale brings amax within the codes' range."""
    up = (amax.view(torch.int32) + 0x1FFFFF) >> 23                        # exponent field, one more past 1.75
    return (up - CODE_TOP[code]).clamp(min=EXP_MIN, max=EXP_MAX[code])


def _encode(x, e, code):
    top = CODE_MAX[code]
    return (x * _power(254 - e)).clamp(min=-top, max=top).to(CODES[code]).view(torch.uint8)


def _query(s):
    case = s["case"]
    if s["q"] is None:
        return None
    return _turned(s["q"], _positions(s), s["freq"], case["interleaved"], 0, case["magnitude"]).to(TYPES[case["type"]])


def _kv_store(s):
    """A page's scale is the least power of two that holds its values; where new ones need a larger one, the old are rounded again."""
    case = s["case"]
    page, code = case["page"], case["code"]
    k = _turned(s["k"], _positions(s), s["freq"], case["interleaved"], 0, case["magnitude"])
    row, rows = s["runs"].long().unbind(1)
    rows = torch.where(torch.arange(row.numel(), device=row.device) < s["counts"][1], rows, 0)
    slot = s["slots"][row]
    at = torch.where(rows > 0, slot // page, s["k_exp"].shape[0] - 1)     # other runs write the spare page's own bytes back
    offset = (slot % page)[:, None]
    pos = torch.arange(page, device=row.device)
    is_new = (rows > 0)[:, None] & (pos >= offset) & (pos < offset + rows[:, None])
    is_old = (rows > 0)[:, None] & (pos < offset)
    take = (row[:, None] + pos - offset).clamp(min=0, max=s["tokens"] - 1)
    _store_one(k, s["k_cache"], s["k_exp"], at, take, is_new, is_old, code, False)
    _store_one(s["v"], s["v_cache"], s["v_exp"], at, take, is_new, is_old, code, True)
    return _kv_result(s, _query(s))


def _store_one(x, cache, exps, at, take, is_new, is_old, code, across):
    x = x[take].permute(0, 2, 1, 3).float()                               # [runs, kv, page, dim]
    is_new, is_old = is_new[:, None, :, None], is_old[:, None, :, None]
    amax = torch.where(is_new, x.abs(), 0.0).amax(dim=(2, 3))
    was = torch.where(is_old.any(dim=2)[:, :, 0], exps[at].to(torch.int32), EXP_MIN)
    e = torch.maximum(_exponent(amax, code), was)
    held = cache[at].transpose(2, 3) if across else cache[at]
    old = held.contiguous().view(CODES[code]).float() * _power(was)[:, :, None, None]
    again = is_old & (e > was)[:, :, None, None]
    codes = _encode(torch.where(is_new, x, old), e[:, :, None, None], code)
    codes = torch.where(is_new | again, codes, held)
    cache[at] = codes.transpose(2, 3) if across else codes
    exps[at] = torch.where(is_new.any(dim=2)[:, :, 0], e, exps[at].to(torch.int32)).to(torch.uint8)


def _latent_codes(x, latent, code):
    """Codes and exponents of rows [..., latent + rotary]: one scale for each row and part."""
    ec, er = _exponent(x[..., :latent].abs().amax(dim=-1), code), _exponent(x[..., latent:].abs().amax(dim=-1), code)
    codes = torch.cat([_encode(x[..., :latent], ec[..., None], code), _encode(x[..., latent:], er[..., None], code)], dim=-1)
    return codes, torch.stack([ec, er], dim=-1).to(torch.uint8)


def _latent_store(s):
    case = s["case"]
    turned = _turned(s["k_rot"][:, None], _positions(s), s["freq"], case["interleaved"], 0, case["magnitude"])[:, 0]
    codes, exps = _latent_codes(torch.cat([s["latent"].float(), turned], dim=-1), case["latent"], case["code"])
    at, place = s["slots"] // case["page"], s["slots"] % case["page"]
    s["codes"][at, place] = codes
    s["exps"][at, place] = exps
    return _latent_result(s, _query(s))


def _latent(s):
    case = s["case"]
    page, code, latent, heads = case["page"], case["code"], case["latent"], case["heads"]
    lens, start = s["lens"].long(), s["q_start"].long()
    new = start[1:] - start[:-1]
    n, longest, rows = new.numel(), s["table"].shape[1] * page, s["max_new"]
    pages = s["table"].clamp(min=0).long()
    x = s["codes"].view(CODES[code])[pages].float()
    scale = _power(s["exps"])[pages]
    c = (x[..., :latent] * scale[..., :1]).view(n, longest, latent)
    keys = torch.cat([c, (x[..., latent:] * scale[..., 1:]).view(n, longest, case["rot"])], dim=-1)
    j = torch.arange(rows, device=lens.device)
    t = torch.arange(longest, device=lens.device)
    take = (start[:-1, None] + j).clamp(max=s["tokens"] - 1)
    q = s["q"][take].float().view(n, rows * heads, -1)
    seen = t <= ((lens - new)[:, None] + j)[:, :, None]
    seen = seen & (t < lens[:, None, None])
    scores = (torch.matmul(q, keys.transpose(1, 2)) * s["scale"]).view(n, rows, heads, longest).masked_fill_(~seen[:, :, None], -math.inf)
    return _attended(s, scores, c, torch.searchsorted(start[1:].contiguous(), torch.arange(s["tokens"], device=lens.device), right=True))


def _attended(s, scores, values, i):
    """softmax(scores) values, scores [requests, rows, heads, tokens]; then the rows in their order, each of request i."""
    n, rows, heads, _ = scores.shape
    top = scores.amax(dim=-1, keepdim=True)
    scores = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = scores.sum(dim=-1, keepdim=True)
    if values.dim() == 3:                                                 # the same for all heads
        out = torch.matmul(scores.view(n, rows * heads, -1), values).view(n, rows, heads, -1)
    else:
        out = torch.matmul(scores.transpose(1, 2), values).transpose(1, 2)
    out = out / torch.where(total > 0, total, 1.0)
    at = torch.arange(s["tokens"], device=i.device) - s["q_start"].long()[i]
    return {"out": out[i, at].to(TYPES[s["case"]["type"]]), "lse": (top + torch.log(total))[i, at, :, 0]}


def _expanded(s):
    case = s["case"]
    start, begin = s["q_start"].long(), s["k_start"].long()
    new, lens = start[1:] - start[:-1], begin[1:] - begin[:-1]
    n, rows, longest = new.numel(), s["max_new"], s["max_len"]
    j, t = torch.arange(rows, device=new.device), torch.arange(longest, device=new.device)
    take = (start[:-1, None] + j).clamp(max=s["tokens"] - 1)
    held = (begin[:-1, None] + t).clamp(max=s["k"].shape[0] - 1)
    q = s["q"][take].float().transpose(1, 2)                              # [requests, heads, rows, .]
    k, v = s["k"][held].float().transpose(1, 2), s["v"][held].float().transpose(1, 2)
    nope = case["nope"]
    scores = torch.matmul(q[..., :nope], k.transpose(2, 3)) + torch.matmul(q[..., nope:], s["k_rot"][held].float().transpose(1, 2)[:, None])
    seen = t <= ((lens - new)[:, None] + j)[:, :, None]
    seen = seen & (t < lens[:, None, None])
    scores = (scores * s["scale"]).masked_fill_(~seen[:, None], -math.inf).transpose(1, 2)
    return _attended(s, scores, v, torch.searchsorted(start[1:].contiguous(), torch.arange(s["tokens"], device=new.device), right=True))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = SIZES[case["type"]]
    if case["op"] == "rotate":
        rows, values = case["rows"], case["rows"] * case["heads"]
        return {"bytes": 2 * values * case["dim"] * size + 4 * rows + 2 * case["rot"], "flops": 3 * values * case["rot"]}
    ctx, new = _lengths(case)
    tokens, heads, reqs = _tokens(case), case["heads"], len(ctx)
    small = 8 * reqs + 4 + 8 * tokens
    if case["op"] == "kv_store":
        runs = sum((c + n - 1) // case["page"] - c // case["page"] + 1 for c, n in zip(ctx, new))
        kv, dim = case["kv"], case["dim"]
        return {"bytes": 2 * tokens * kv * dim * (size + 1) + 2 * tokens * heads * dim * size + 2 * runs * kv + 16 * runs + small,
                "flops": 3 * tokens * (heads + kv) * case["rot"]}
    rot = case["rot"]
    if case["op"] == "latent_store":
        return {"bytes": tokens * (case["latent"] + rot) * (size + 1) + 2 * tokens + 2 * tokens * heads * rot * size + small,
                "flops": 3 * tokens * (heads + 1) * rot}
    pairs = sum(c * n + n * (n + 1) // 2 for c, n in zip(ctx, new))
    held = sum(ctx) + tokens
    if case["op"] == "latent":
        latent = case["latent"]
        return {"bytes": held * (latent + rot + 2) + tokens * heads * ((2 * latent + rot) * size + 4) + 4 * (held // case["page"] + reqs) + 8 * reqs,
                "flops": 2 * pairs * heads * (2 * latent + rot)}
    nope, value = case["nope"], case["value"]
    return {"bytes": held * (heads * (nope + value) + rot) * size + tokens * heads * ((nope + rot + value) * size + 4) + 8 * reqs,
            "flops": 2 * pairs * heads * (nope + rot + value)}


# ------------------------------------------------------------------ the definitions in 64 bits
def _two(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _as_values(codes, code):
    """Codes as the numbers they stand for, from their bits."""
    c = codes.long()
    bits, bias = (3, 7) if code == "e4m3fn" else (2, 15)
    field, frac = (c >> bits) & ((1 << (7 - bits)) - 1), (c & ((1 << bits) - 1)).double() / (1 << bits)
    x = torch.where(field > 0, (1 + frac) * _two(field - bias), frac * 2.0 ** (1 - bias))
    return torch.where(c >= 128, -x, x)


def _rounded(x, code):
    """x to the nearest number that the code has, ties to the even one; past its range the largest."""
    x = x.clamp(min=-CODE_MAX[code], max=CODE_MAX[code])
    bits, low = (3, -6) if code == "e4m3fn" else (2, -14)
    ulp = _two((torch.frexp(x).exponent.long() - 1).clamp(min=low) - bits)
    return torch.round(x / ulp) * ulp


def _least_power(most, code):
    """The least e with most <= the largest code times 2^e, within the exponent byte's range."""
    small = torch.frexp(most / CODE_MAX[code])
    e = torch.where(most > 0, small.exponent.long() - (small.mantissa == 0.5).long(), EXP_MIN - 127)
    return e.clamp(min=EXP_MIN - 127, max=EXP_MAX[code] - 127)


def _turned_exactly(x, positions, freq, interleaved, first, magnitude, inverse=False):
    """Each pair as a complex number, times e^(i angle)."""
    x = x.double()
    half = freq.numel()
    angle = positions.double()[:, None, None] * freq.double() * (-1 if inverse else 1)
    pairs = torch.arange(half, device=x.device)
    a, b = (first + 2 * pairs, first + 2 * pairs + 1) if interleaved else (first + pairs, first + half + pairs)
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full_like(angle, magnitude), angle)
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _places_exactly(s):
    lens, start = s["lens"].tolist(), s["q_start"].tolist()
    return torch.cat([torch.arange(n - (b - a), n, device=DEVICE) for n, a, b in zip(lens, start, start[1:])])


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotate":
        return _turned_exactly(s["x"], s["positions"], s["freq"], case["interleaved"], case["first"], case["magnitude"], case["inverse"])
    if op == "latent":
        return _latent_exactly(case, s)
    if op == "expanded":
        return _expanded_exactly(case, s)
    code, page, at = case["code"], case["page"], _places_exactly(s)
    turn = (s["freq"], case["interleaved"], 0, case["magnitude"])
    if op == "latent_store":
        latent = case["latent"]
        x = torch.cat([s["latent"].double(), _turned_exactly(s["k_rot"][:, None], at, *turn)[:, 0]], dim=-1)
        codes, exps = _as_values(s["codes"], code), s["exps"].clone()
        for part, which in enumerate((slice(0, latent), slice(latent, None))):
            e = _least_power(x[:, which].abs().amax(dim=1), code)
            codes.view(-1, codes.shape[2])[s["slots"], which] = _rounded(x[:, which] * _two(-e)[:, None], code)
            exps.view(-1, 2)[s["slots"], part] = (e + 127).to(torch.uint8)
        done = {"codes": codes, "exps": exps}
    else:
        slots, done = s["slots"].tolist(), {}
        for name in ("k", "v"):
            x = _turned_exactly(s["k"], at, *turn) if name == "k" else s["v"].double()
            cache = s["k_cache"] if name == "k" else s["v_cache"].transpose(2, 3)
            value = _as_values(cache, code)
            exps = s[name + "_exp"].long() - 127
            for first, n in s["runs"].tolist()[:int(s["counts"][1])]:
                p, offset = divmod(slots[first], page)
                new = x[first:first + n].transpose(0, 1)                  # [kv, n, dim]
                e = _least_power(new.abs().amax(dim=(1, 2)), code)
                if offset:
                    was = exps[p].clone()
                    e = torch.maximum(e, was)
                    value[p, :, :offset] = _rounded(value[p, :, :offset] * _two(was - e)[:, None, None], code)
                exps[p] = e
                value[p, :, offset:offset + n] = _rounded(new * _two(-e)[:, None, None], code)
            done[name] = value if name == "k" else value.transpose(2, 3).contiguous()
            done[name + "_exp"] = (exps + 127).to(torch.uint8)
        done = {key: done[key] for key in ("k", "v", "k_exp", "v_exp")}
    if s["q"] is not None:
        done["q"] = _turned_exactly(s["q"], at, *turn)
    return done


def _softmax_rows(q, keys, values, places, scale):
    """Of one head: each row over the tokens up to its place."""
    z = (q @ keys.T) * scale
    z = torch.where(torch.arange(keys.shape[0], device=DEVICE) <= places[:, None], z, -math.inf)
    return torch.softmax(z, dim=1) @ values, torch.logsumexp(z, dim=1)


def _latent_exactly(case, s):
    page, latent, heads = case["page"], case["latent"], case["heads"]
    out = torch.zeros(s["tokens"], heads, latent, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(s["tokens"], heads, dtype=torch.float64, device=DEVICE)
    lens, start = s["lens"].tolist(), s["q_start"].tolist()
    for i, length in enumerate(lens):
        a, b = start[i], start[i + 1]
        pages = s["table"][i, :-(-length // page)].long()
        keys, exps = _as_values(s["codes"][pages], case["code"]).flatten(0, 1)[:length], s["exps"][pages].flatten(0, 1)[:length].long()
        keys[:, :latent] *= _two(exps[:, :1] - 127)
        keys[:, latent:] *= _two(exps[:, 1:] - 127)
        places = torch.arange(length - (b - a), length, device=DEVICE).repeat_interleave(heads)
        q, step = s["q"][a:b].double().flatten(0, 1), max(1, (1 << 26) // length)
        o, e = out[a:b].view(-1, latent), lse[a:b].view(-1)
        for r in range(0, q.shape[0], step):
            o[r:r + step], e[r:r + step] = _softmax_rows(q[r:r + step], keys, keys[:, :latent], places[r:r + step], s["scale"])
    return {"out": out, "lse": lse}


def _expanded_exactly(case, s):
    out = torch.zeros(s["tokens"], case["heads"], case["value"], dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(s["tokens"], case["heads"], dtype=torch.float64, device=DEVICE)
    start, begin = s["q_start"].tolist(), s["k_start"].tolist()
    for i in range(case["reqs"]):
        a, b, c, d = start[i], start[i + 1], begin[i], begin[i + 1]
        places = torch.arange(d - c - (b - a), d - c, device=DEVICE)
        for h in range(case["heads"]):
            keys = torch.cat([s["k"][c:d, h], s["k_rot"][c:d]], dim=-1).double()
            out[a:b, h], lse[a:b, h] = _softmax_rows(s["q"][a:b, h].double(), keys, s["v"][c:d, h].double(), places, s["scale"])
    return {"out": out, "lse": lse}
