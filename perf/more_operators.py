"""The performance cases of the 4-bit paged cache: what a serving program with long contexts asks of it.

A cache element takes 4 bits and its share of a scale: E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a
byte with the even element low, and for 32 neighbouring elements of a head one byte b for the scale 2^(b - 127), the
least power of two s with max |x| <= 7 s. Four calls work on it:

  rope     norms of queries and keys for each head, rotation, keys and values into their slots in 4 bits
  attend   attention over the pages, and the logarithm of each row's sum for the next call
  weigh    the attention weight that every key of every cache head has got, added up over queries
  evict    each cache head keeps the heaviest keys of a request, first and last ones aside; pages come back

Sizes come from the configurations, tests and benchmark of this repository (blocks of 16, 1 to 256 requests, heads of
128) or are generic; contexts are longer than a 16-bit cache's cases have them. Lengths follow a fixed low-discrepancy
pattern, so that a case's work is known without its inputs; values and the order of the pages come from the seed.
Codes and scales come back as they lie in the cache, as whole numbers: the nearest code of the exact value is the only
right one, and a cache that has been cut holds the kept tokens' very bytes.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
SPARE = 7  # pages in every cache that no table lists


def _named(name, c):
    return dict(c, name=name) if name else c


def _rope(name, T, Hq, Hkv, D, rot, page, dtype="bf16", interleaved=False, norm=True):
    return _named(name, {"kind": "rope", "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "page": page,
                         "dtype": dtype, "interleaved": interleaved, "norm": norm})


def _attend(name, N, lo, hi, ctx_lo, ctx_hi, Hq, Hkv, D, page, window=0, sinks=0, dtype="bf16", causal=True):
    """lo .. hi new tokens and ctx_lo .. ctx_hi tokens in the cache before them, per request."""
    return _named(name, {"kind": "attend", "N": N, "lo": lo, "hi": hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "Hq": Hq,
                         "Hkv": Hkv, "D": D, "page": page, "window": window, "sinks": sinks, "dtype": dtype,
                         "causal": causal})


def _weigh(name, N, lo, hi, ctx_lo, ctx_hi, Hq, Hkv, D, page, decay=1.0, dtype="bf16"):
    return _named(name, {"kind": "weigh", "N": N, "lo": lo, "hi": hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "Hq": Hq,
                         "Hkv": Hkv, "D": D, "page": page, "window": 0, "sinks": 0, "decay": decay, "dtype": dtype,
                         "causal": True})


def _evict(name, N, len_lo, len_hi, Hkv, D, page, budget, limit, sinks, recent):
    return _named(name, {"kind": "evict", "N": N, "len_lo": len_lo, "len_hi": len_hi, "Hkv": Hkv, "D": D,
                         "page": page, "budget": budget, "limit": limit, "sinks": sinks, "recent": recent})


def listed():
    return [
        # one user, one token: nothing but latency
        _rope("rope one token", 1, 32, 8, 128, 128, 16),
        # a step full of prefill chunks
        _rope("rope prefill", 16381, 32, 8, 128, 128, 64),
        # nothing is a round number: heads of 96, a third of each rotated, neighbouring pairs, fp16
        _rope("rope odd fp16", 2777, 15, 5, 96, 32, 24, dtype="fp16", interleaved=True),
        # one user, one token, a long conversation
        _attend("attend one token", 1, 1, 1, 32767, 32767, 32, 8, 128, 16),
        # a full server, one token each: the largest read
        _attend("attend 256 tokens", 256, 1, 1, 100, 16100, 32, 8, 128, 64),
        # the benchmark's batch: the target checks 64 blocks of 16 drafted tokens
        _attend("attend 64 blocks", 64, 16, 16, 1000, 16000, 32, 8, 128, 16),
        # a prefill chunk behind a long context: matrix work
        _attend("attend prefill", 1, 8192, 8192, 8192, 8192, 32, 8, 128, 16),
        # odd: blocks of any length, none among them, seen from both sides behind a window, odd pages, heads of 64
        _attend("attend ragged fp16", 37, 0, 33, 0, 5000, 14, 2, 64, 24, window=1000, sinks=7, dtype="fp16",
                causal=False),
        # the keys of a long conversation after one token of a full server
        _weigh("weigh 256 tokens", 256, 1, 1, 100, 16100, 32, 8, 128, 64, decay=0.98),
        # a prompt's last chunk says which keys of the prompt count
        _weigh("weigh prompt", 1, 1024, 1024, 31744, 31744, 32, 8, 128, 16),
        # one long conversation is cut to an eighth
        _evict("evict one", 1, 32768, 32768, 8, 128, 16, 4096, 4096, 4, 256),
        # a full server: most requests are over the limit, of any length
        _evict("evict 64 ragged", 64, 500, 16000, 8, 128, 64, 2500, 3000, 5, 333),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choices(("rope", "attend", "weigh", "evict"), (2, 5, 3, 3))[0]
        page = rng.choice((8, 16, 16, 16, 24, 32, 64, 128))
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        Hkv, G = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 6, 8))
        D = rng.choice((64, 64, 96, 128, 128, 128, 256))
        form = rng.choice(("token", "block", "block", "ragged", "prefill"))
        N = _log(rng, 1, 256)
        lo, hi = {"token": (1, 1), "block": (16, 16), "ragged": (0, _log(rng, 2, 300)),
                  "prefill": (1, _log(rng, 200, 8192))}[form]
        if form == "prefill":
            N = max(1, N // 32)
        ctx = _log(rng, 16, 32767)
        least = rng.choice((0, ctx // 8, ctx))
        if kind == "rope":
            c = _rope(None, _log(rng, 1, 16381), Hkv * G, Hkv, D, 16 * rng.randint(1, D // 16), page, dtype,
                      rng.random() < 0.3, rng.random() < 0.8)
        elif kind == "attend":
            window, sinks = (_log(rng, 128, 4096), rng.choice((0, 1, 4, 4, 7, 64))) if rng.random() < 0.3 else (0, 0)
            c = _attend(None, N, lo, hi, least, ctx, Hkv * G, Hkv, D, page, window, sinks, dtype, rng.random() < 0.8)
        elif kind == "weigh":
            c = _weigh(None, N, lo, hi, least, ctx, Hkv * G, Hkv, D, page, rng.choice((1.0, 0.98, 0.5)), dtype)
        else:
            most = _log(rng, 200, 32768)
            budget = _log(rng, 64, min(8192, most))
            sinks, recent = rng.choice((0, 1, 4, 7)), rng.choice((0, 1, budget // 8, budget // 3))
            c = _evict(None, max(1, N // 4), most // rng.choice((1, 8, 50)), most, Hkv, D, page, budget,
                       budget + rng.choice((0, 0, budget // 5)), sinks, recent)
        # no dearer than the largest listed cases, and a plain form that fits the card
        w = work(c)
        if w["bytes"] > 2.2e9 or w["flops"] > 1.6e12:
            continue
        if kind in ("attend", "weigh"):
            new, _, total = _lengths(c)
            if max(new) * c["N"] * c["Hq"] * max(total) > 4.2e9 or c["N"] * max(total) * c["Hkv"] * D > 4.3e9:
                continue
            if sum(new) == 0:
                continue
        if kind == "evict" and c["N"] * max(c["len_hi"], c["budget"]) * c["Hkv"] * D > 2.2e9:
            continue
        return c


# ---- lengths and work ------------------------------------------------------------------------------

def _spread(n, lo, hi, step):
    return lo + int((n * step + 0.37) % 1.0 * (hi - lo + 1))


def _lengths(c):
    """(new tokens, tokens before them, both) of every request; the first one takes the most."""
    N = c["N"]
    new = [c["hi"] if n == 0 else _spread(n, c["lo"], c["hi"], 0.61803398875) for n in range(N)]
    ctx = [c["ctx_hi"] if n == 0 else _spread(n, c["ctx_lo"], c["ctx_hi"], 0.7548776662) for n in range(N)]
    return new, ctx, [a + b for a, b in zip(new, ctx)]


def _held(c):
    """Tokens of every request before an eviction; the first one takes the most."""
    return [c["len_hi"] if n == 0 else _spread(n, c["len_lo"], c["len_hi"], 0.7548776662) for n in range(c["N"])]


def _visible(p, total, c):
    """Keys that the query at position p sees."""
    hi = min(total, p + 1) if c["causal"] else total
    if not c["window"]:
        return max(0, hi)
    lo = max(0, p - c["window"] + 1)
    return max(0, hi - lo) + min(c["sinks"], lo, max(hi, 0))


def work(case):
    c = case
    if c["kind"] == "rope":  # queries in and out, keys and values in, and out in 17/32 of a byte an element
        return {"bytes": c["T"] * (c["Hq"] * c["D"] * 4 + 2 * c["Hkv"] * (c["D"] * 2 + c["D"] * 17 // 32) +
                                   c["rot"] * 4 + 8),
                "flops": c["T"] * (c["Hq"] + c["Hkv"]) * c["D"] * 7}
    row = c["D"] * 17 // 32  # bytes of a key, or value, of one head
    if c["kind"] == "evict":
        over = [t for t in _held(c) if t > c["limit"]]
        moved = len(over) * (c["budget"] - c["sinks"])
        return {"bytes": c["Hkv"] * (4 * sum(over) + moved * 2 * (2 * row + 4)) + 20 * c["N"] +
                         8 * sum((t - c["budget"]) // c["page"] for t in over) + 1, "flops": 0}
    new, ctx, total = _lengths(c)
    pairs = keys = 0
    for t, x, n in zip(new, ctx, total):
        if not t:
            continue
        mid = [_visible(x + round(k * (t - 1) / 32), n, c) for k in range(33)] if t > 33 else \
            [_visible(x + k, n, c) for k in range(t)]
        pairs += t * sum(mid) / len(mid)
        seen = n if not c["window"] else n - max(0, x - c["window"] + 1) + min(c["sinks"], max(0, x - c["window"] + 1))
        keys += seen
    rows = sum(new) * c["Hq"]
    if c["kind"] == "weigh":
        return {"bytes": keys * c["Hkv"] * (row + 8) + rows * (c["D"] * 2 + 4) + keys * 4 // c["page"],
                "flops": 2 * pairs * c["Hq"] * c["D"]}
    return {"bytes": keys * c["Hkv"] * 2 * row + rows * (c["D"] * 4 + 4) + keys * 4 // c["page"],
            "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed, tag):
    return torch.Generator(device="cuda").manual_seed((seed * 1_000_003 + tag) & ((1 << 62) - 1))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _to4(x):
    """[.., d] -> codes [.., d / 2] and scales [.., d / 32], both uint8. Finite values; exact for every type."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    most = b.abs().amax(-1)
    m, e = torch.frexp(most)  # most = m 2^e with m in [0.5, 1)
    e = torch.where(most == 0, -200, e - torch.where(m <= 0.875, 3, 2)).clamp(-126, 125)
    v = torch.ldexp(b.abs().double(), -e[..., None]).to(torch.float64 if x.dtype == torch.float64 else torch.float32)
    # steps end half-way between two values; a tie goes to the one whose code is even
    code = (v > 0.25).byte() + (v >= 0.75).byte() + (v > 1.25).byte() + (v >= 1.75).byte() + (v > 2.5).byte() + \
        (v >= 3.5).byte() + (v > 5).byte() + torch.signbit(b).byte() * 8
    code = code.reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | code[..., 1] << 4, (e + 127).to(torch.uint8)


def _from4(codes, scales):
    """What codes [.., d / 2] and scales [.., d / 32] stand for: fp32 [.., d]."""
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    both = torch.stack((value[(codes & 15).long()], value[(codes >> 4).long()]), -1)
    x = both.reshape(*codes.shape[:-1], -1, 32) * torch.exp2(scales.float() - 127)[..., None]
    return x.reshape(*codes.shape[:-1], -1)


def _cache(pages, P, Hkv, D, g, scale=1.0):
    """Codes and scales of normal values, made a piece at a time."""
    rows = pages * P * Hkv
    codes = torch.empty(rows, D // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, D // 32, dtype=torch.uint8, device="cuda")
    step = (1 << 26) // D
    for at in range(0, rows, step):
        n = min(step, rows - at)
        codes[at:at + n], scales[at:at + n] = _to4(torch.randn(n, D, generator=g, device="cuda").mul_(scale))
    return codes.view(pages, P, Hkv, D // 2), scales.view(pages, P, Hkv, D // 32)


def _tables(counts, width, order):
    """Table [N, width] whose row n lists the next counts[n] pages of `order`, -1 after them."""
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for n, k in enumerate(counts):
        table[n, :k] = order[at:at + k]
        at += k
    return table


def _prepare_rope(c, seed):
    T, Hq, Hkv, D, rot, P = (c[k] for k in ("T", "Hq", "Hkv", "D", "rot", "page"))
    g, dtype = _generator(seed, 12), DTYPE[c["dtype"]]
    # one projection's output, of which queries, keys and values are views
    qkv = (torch.randn(T, (Hq + 2 * Hkv) * D, generator=g, device="cuda") * 1.5).to(dtype)
    pages = -(-T // P) * 2 + SPARE
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:T].to(torch.int32)
    slots[torch.rand(T, generator=g, device="cuda") < 0.01] = -1  # tokens that have no page
    most = 32768
    angle = torch.arange(most, device="cuda", dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) / (rot // 2))
    s = {"c": c, "q": qkv[:, :Hq * D].view(T, Hq, D),
         "k": qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D), "v": qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D),
         "slots": slots, "positions": torch.randint(0, most, (T,), generator=g, device="cuda").to(torch.int32),
         "cos_sin": torch.cat((angle.cos(), angle.sin()), 1).float(),
         "k4": _cache(pages, P, Hkv, D, g), "v4": _cache(pages, P, Hkv, D, g),
         "q_weight": None, "k_weight": None, "out": torch.empty(T, Hq, D, dtype=dtype, device="cuda")}
    if c["norm"]:
        for name in ("q_weight", "k_weight"):
            s[name] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    return s


def _prepare_attend(c, seed):
    N, Hq, Hkv, D, P = (c[k] for k in ("N", "Hq", "Hkv", "D", "page"))
    g, dtype = _generator(seed, 13), DTYPE[c["dtype"]]
    new, _, total = _lengths(c)
    counts = [-(-t // P) for t in total]
    pages = sum(counts) + SPARE
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    starts = [0]
    for t in new:
        starts.append(starts[-1] + t)
    # heads of different sharpness: scores of a standard deviation from 0.5 to 4
    q = torch.randn(starts[-1], Hq, D, generator=g, device="cuda")
    q = (q * (0.5 * 2.0 ** (torch.arange(Hq, device="cuda") % 4))[None, :, None]).to(dtype)
    return {"c": c, "q": q, "k4": _cache(pages, P, Hkv, D, g), "v4": _cache(pages, P, Hkv, D, g),
            "table": _tables(counts, max(counts) + 1, order), "starts": _i32(starts), "totals": _i32(total),
            "out": torch.empty_like(q), "lse": torch.empty(starts[-1], Hq, device="cuda"),
            "most_tokens": max(new), "most_keys": max(total), "workspace": None}


def _prepare_weigh(c, seed):
    """The state after an attention call: its rows' logarithms, and the weights that keys have from earlier steps."""
    s = _prepare_attend(c, seed)
    g, pages = _generator(seed, 14), s["k4"][0].shape[0]
    starts, totals = s["starts"].tolist(), s["totals"].tolist()
    for n, total in enumerate(totals):
        k = _keys_of(s, n, total)
        for t in range(starts[n], starts[n + 1], 256):
            q = s["q"][t:min(t + 256, starts[n + 1])].float()
            p = torch.arange(total - starts[n + 1] + t, total - starts[n + 1] + t + q.shape[0], device="cuda")
            z = q.view(q.shape[0], c["Hkv"], -1, c["D"]).permute(1, 2, 0, 3).flatten(1, 2) @ k.transpose(1, 2)
            z = z.view(c["Hq"], q.shape[0], total) / math.sqrt(c["D"])
            z.masked_fill_(torch.arange(total, device="cuda") > p[:, None], -math.inf)
            s["lse"][t:t + q.shape[0]] = torch.logsumexp(z, -1).T
    del s["v4"]
    # heavy tails: a few keys have got most of the weight
    s["weights"] = torch.empty(pages, c["Hkv"], c["page"], device="cuda").exponential_(generator=g) ** 3
    return s


def _prepare_evict(c, seed):
    N, Hkv, D, P = (c[k] for k in ("N", "Hkv", "D", "page"))
    g = _generator(seed, 15)
    held = _held(c)
    ends = [-(-t // P) + n % 3 for n, t in enumerate(held)]  # some hold pages for tokens that were rejected
    total = sum(ends) + SPARE
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = _tables(ends, max(ends) + 1, order)
    free = order[sum(ends):]
    head = int(torch.randint(0, 5 * total, (1,), generator=g, device="cuda"))
    queue = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    queue[(head + torch.arange(free.numel(), device="cuda")) % total] = free
    weights = torch.empty(total, Hkv, P, device="cuda").exponential_(generator=g) ** 3
    weights[torch.rand(total, Hkv, P, generator=g, device="cuda") < 0.05] = 0.0  # keys that no query has met
    return {"c": c, "k4": _cache(total, P, Hkv, D, g), "v4": _cache(total, P, Hkv, D, g), "weights": weights,
            "table": table, "totals": _i32(held), "pages": _i32([(e, 0) for e in ends]), "queue": queue,
            "cursor": torch.tensor([head, head + free.numel(), 0], device="cuda"), "most_keys": max(held),
            "workspace": None}


def prepare(case, seed):
    return {"rope": _prepare_rope, "attend": _prepare_attend, "weigh": _prepare_weigh,
            "evict": _prepare_evict}[case["kind"]](case, seed)


# ---- one pass --------------------------------------------------------------------------------------

def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), rest), -1)
    a, b = r[..., :rot // 2], r[..., rot // 2:]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)


def _cache_of(s):
    return {"k": s["k4"][0], "k_scales": s["k4"][1], "v": s["v4"][0], "v_scales": s["v4"][1]}


def _plain_rope(s):
    c, dtype = s["c"], s["q"].dtype
    made = []
    # keys in 64 bits: their codes and scales are whole numbers that values next to a border decide
    for x, w, wide in ((s["q"], s["q_weight"], torch.float32), (s["k"], s["k_weight"], torch.float64)):
        cos, sin = s["cos_sin"][s["positions"].long()][:, None].to(wide).chunk(2, -1)
        x = x.to(wide)
        if w is not None:
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w
        made.append(_rotated(x, cos, sin, c["interleaved"]))
    live = s["slots"] >= 0
    at = s["slots"][live].long()
    for cache, x in ((s["k4"], made[1]), (s["v4"], s["v"])):
        for part, y in zip(cache, _to4(x[live])):
            part.view(-1, c["Hkv"], part.shape[-1])[at] = y
    return {"q": made[0].to(dtype), **_cache_of(s)}


def _padded(s):
    """Queries padded to [N, Hkv, most * G, D], with where they come from, and every key's slot [N, keys]."""
    c, q, P = s["c"], s["q"], s["c"]["page"]
    N, Hkv, D, G = c["N"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    dev, most, keys = q.device, s["most_tokens"], s["most_keys"]
    starts, total = s["starts"].long(), s["totals"].long()
    new = starts[1:] - starts[:-1]
    t = torch.arange(most, device=dev)
    live = t < new[:, None]
    at = torch.where(live, starts[:-1, None] + t, 0)
    x = q[at].float().view(N, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(N, Hkv, most * G, D)
    j = torch.arange(keys, device=dev)
    page = s["table"].long()[:, j // P]
    held = (page >= 0) & (j < total[:, None])
    slot = torch.where(held, page * P + j % P, 0)
    p = (total - new)[:, None] + t
    seen = held[:, None, :].expand(N, most, keys)
    if c["causal"]:
        seen = seen & (j <= p[:, :, None])
    if c["window"]:
        seen = seen & ((j > p[:, :, None] - c["window"]) | (j < c["sinks"]))
    return x, at, live, slot, held, new, seen.repeat_interleave(G, 1)[:, None]


def _gathered(cache, slot):
    """fp32 [N, heads, keys, d] of the tokens at slot [N, keys]."""
    codes, scales = (part.flatten(0, 1)[slot].permute(0, 2, 1, 3) for part in cache)
    return _from4(codes, scales)


def _plain_attend(s):
    c = s["c"]
    N, Hkv, D, G, most = c["N"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"], s["most_tokens"]
    x, _, live, slot, _, _, seen = _padded(s)
    scores = torch.matmul(x, _gathered(s["k4"], slot).transpose(2, 3)).mul_(1 / math.sqrt(D))
    scores = scores.masked_fill_(~seen, -math.inf)
    m = scores.amax(-1, keepdim=True)
    scores = scores.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    z = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores, _gathered(s["v4"], slot)) / torch.where(z == 0, 1.0, z)
    o = o.view(N, Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(N, most, Hkv * G, D)
    lse = torch.where(z == 0, -math.inf, m + z.log()).view(N, Hkv, most, G).permute(0, 2, 1, 3).reshape(N, most, -1)
    return {"out": o[live].to(s["q"].dtype), "lse": lse[live]}


def _plain_weigh(s):
    c = s["c"]
    N, Hkv, D, G, most = c["N"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"], s["most_tokens"]
    x, at, live, slot, held, new, seen = _padded(s)
    scores = torch.matmul(x, _gathered(s["k4"], slot).transpose(2, 3)).mul_(1 / math.sqrt(D))
    lse = s["lse"][at].view(N, most, Hkv, G).permute(0, 2, 1, 3).reshape(N, Hkv, most * G, 1)
    seen = seen & live.repeat_interleave(G, 1)[:, None, :, None]
    got = scores.sub_(lse).exp_().masked_fill_(~seen, 0.0).sum(2)  # [N, Hkv, keys]
    P = c["page"]
    place = (slot // P)[:, None], torch.arange(Hkv, device=slot.device)[:, None], (slot % P)[:, None]
    j = torch.arange(slot.shape[1], device=slot.device)
    before = (j < (s["totals"].long() - new)[:, None])[:, None]  # keys of earlier steps have a weight already
    w = torch.where(before, s["weights"][place] * c["decay"], 0.0) + got
    there = (held & (new > 0)[:, None])[:, None].expand_as(w)
    s["weights"][tuple(i.expand_as(w)[there] for i in place)] = w[there]
    return {"weights": s["weights"]}


def _plain_evict(s):
    c, P, M, C = s["c"], s["c"]["page"], s["table"].shape[1], s["queue"].numel()
    N, Hkv, B, keys = c["N"], c["Hkv"], c["budget"], s["most_keys"]
    dev = s["table"].device
    length, end = s["totals"].long(), s["pages"][:, 0].long()
    cut = length > c["limit"]
    after = torch.where(cut, B, length)
    left = torch.where(cut, -(-after // P), end)
    give = end - left
    gave = give.cumsum(0) - give
    tail = s["cursor"][1]
    n = torch.repeat_interleave(give)
    r = torch.arange(n.numel(), device=dev) - gave[n]
    s["queue"][(tail + gave[n] + r) % C] = s["table"][n, left[n] + r]
    out = {"totals": after.to(torch.int32),
           "pages": torch.stack((left, s["pages"][:, 1].long()), 1).to(torch.int32),
           "cursor": torch.stack((s["cursor"][0], tail + give.sum(), s["cursor"][2])),
           "evicted": (length - after).to(torch.int32)}
    if keys > B:
        j = torch.arange(keys, device=dev)
        slot = s["table"].long()[:, (j // P).clamp(max=M - 1)].clamp(min=0) * P + j % P
        place = (slot // P)[:, None], torch.arange(Hkv, device=dev)[:, None], (slot % P)[:, None]
        w = s["weights"][place].double()  # [N, Hkv, keys]
        w = w.masked_fill(((j < c["sinks"]) | (j >= length[:, None] - c["recent"]))[:, None], math.inf)
        w = w.masked_fill((j >= length[:, None])[:, None], -math.inf)
        first = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :B]  # ties: the earliest
        first = first.sort(-1).values  # [N, Hkv, B]
        chosen = cut[:, None, None].expand_as(first)
        h = torch.arange(Hkv, device=dev)[:, None].expand_as(first)[chosen]
        source = slot[:, None].expand(N, Hkv, keys).gather(2, first)[chosen]
        to = slot[:, None, :B].expand_as(first)[chosen]
        for part in s["k4"] + s["v4"]:
            flat = part.flatten(0, 1)
            flat[to, h] = flat[source, h]
        s["weights"][to // P, h, to % P] = s["weights"][source // P, h, source % P]
    return {**out, **_cache_of(s), "weights": s["weights"], "queue": s["queue"]}


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"rope": _plain_rope, "attend": _plain_attend, "weigh": _plain_weigh,
                "evict": _plain_evict}[c["kind"]](s)
    import paper_2608_20530_amd as L
    if c["kind"] == "weigh":
        cache = L.Cache4(*s["k4"], None, None)
        return {"weights": L.key_weights(s["q"], s["lse"], cache, s["table"], s["starts"], s["totals"], s["weights"],
                                         decay=c["decay"], max_tokens=s["most_tokens"], max_length=s["most_keys"])}
    cache = L.Cache4(*s["k4"], *s["v4"])
    if c["kind"] == "rope":
        q = L.qk_norm_rope4(s["q"], s["k"], s["v"], s["slots"], s["positions"], s["cos_sin"], cache,
                            q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=c["interleaved"],
                            out=s["out"])
        return {"q": q, **_cache_of(s)}
    if c["kind"] == "attend":
        sizes = {"window": c["window"], "sinks": c["sinks"], "causal": c["causal"], "max_tokens": s["most_tokens"],
                 "max_length": s["most_keys"]}
        if s["workspace"] is None:  # made by the first pass and kept
            s["workspace"] = L.window_attention4_workspace(s["q"], cache, s["table"], **sizes)
        out = L.window_attention4(s["q"], cache, s["table"], s["starts"], s["totals"], lse=s["lse"], out=s["out"],
                                  workspace=s["workspace"], **sizes)
        return {"out": out, "lse": s["lse"]}
    if s["workspace"] is None:
        s["workspace"] = L.evict_workspace(cache, s["table"], budget=c["budget"], max_length=s["most_keys"])
    e = L.evict(cache, s["weights"], s["table"], s["totals"], s["pages"], s["queue"], s["cursor"],
                budget=c["budget"], limit=c["limit"], sinks=c["sinks"], recent=c["recent"],
                max_length=s["most_keys"], workspace=s["workspace"])
    return {"totals": e.totals, "pages": e.pages, "cursor": e.cursor, "evicted": e.evicted, **_cache_of(s),
            "weights": s["weights"], "queue": s["queue"]}


# ---- the definition in 64 bits ---------------------------------------------------------------------

def _read4(codes, scales):
    """Element by element: sign, and 2^e (1 + f / 2), or f / 2 where the exponent's bits are zero."""
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    e, f = (n >> 1) & 3, (n & 1).double() / 2
    x = torch.where(e == 0, f, (1 + f) * 2.0 ** (e - 1).double())
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.long() - 127)
    return torch.where(n > 7, -x, x) * scale.repeat_interleave(32, -1)


def _rows_of(s, n, length):
    at = torch.arange(length, device="cuda")
    return s["table"][n].long()[at // s["c"]["page"]] * s["c"]["page"] + at % s["c"]["page"]


def _keys_of(s, n, length):
    """fp32 keys [Hkv, length, D] of request n."""
    return _from4(*(part.flatten(0, 1)[_rows_of(s, n, length)] for part in s["k4"])).transpose(0, 1)


def _exact_rope(s):
    """Each pair as a complex number, turned by its angle's; a head is normed by its 2-norm."""
    c = s["c"]
    half = c["rot"] // 2
    table = s["cos_sin"].double()
    turn = torch.complex(table[:, :half], table[:, half:])[s["positions"].long()][:, None]
    x = s["q"].double()
    if s["q_weight"] is not None:
        norm = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
        x = x / (norm * norm / c["D"] + EPS).sqrt() * s["q_weight"].double()
    x = x.clone()
    pairs = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else \
        (slice(0, half), slice(half, c["rot"]))
    z = torch.complex(x[..., pairs[0]], x[..., pairs[1]]) * turn
    x[..., pairs[0]], x[..., pairs[1]] = z.real, z.imag
    return {"q": x, **{name: None for name in _cache_of(s)}}  # codes and scales are whole numbers


def _hidden(c, total, new, b, count):
    at = torch.arange(total, device="cuda")[None]
    p = torch.arange(total - new + b, total - new + b + count, device="cuda")[:, None]
    hidden = (at > p) if c["causal"] else torch.zeros_like(at > p)
    if c["window"]:
        hidden = hidden | ((at <= p - c["window"]) & (at >= c["sinks"]))
    return hidden


def _exact_attend(s):
    """Request by request and head by head."""
    c = s["c"]
    G = c["Hq"] // c["Hkv"]
    starts, totals = s["starts"].tolist(), s["totals"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for n, total in enumerate(totals):
        new = starts[n + 1] - starts[n]
        if not new:
            continue
        rows = _rows_of(s, n, total)
        k, v = (_read4(*(part.flatten(0, 1)[rows] for part in s[m])) for m in ("k4", "v4"))  # [keys, Hkv, D]
        q = s["q"][starts[n]:starts[n + 1]].double()
        step = max(1, (1 << 27) // total)
        for b in range(0, new, step):
            count = min(step, new - b)
            hidden = _hidden(c, total, new, b, count)
            for h in range(c["Hq"]):
                z = (q[b:b + count, h] @ k[:, h // G].T) / c["D"] ** 0.5
                z[hidden] = -math.inf
                at = starts[n] + b
                lse[at:at + count, h] = torch.logsumexp(z, 1)
                e = (z - lse[at:at + count, h, None]).exp()
                out[at:at + count, h] = torch.nan_to_num(e) @ v[:, h // G]
    return {"out": out, "lse": lse}


def _exact_weigh(s):
    c = s["c"]
    G, P = c["Hq"] // c["Hkv"], c["page"]
    starts, totals = s["starts"].tolist(), s["totals"].tolist()
    weights = s["weights"].double()
    for n, total in enumerate(totals):
        new = starts[n + 1] - starts[n]
        if not new:
            continue
        rows = _rows_of(s, n, total)
        k = _read4(*(part.flatten(0, 1)[rows] for part in s["k4"]))
        q = s["q"][starts[n]:starts[n + 1]].double()
        w = weights[rows // P, :, rows % P] * c["decay"]  # [total, Hkv]
        w[total - new:] = 0
        hidden = _hidden(c, total, new, 0, new)
        for h in range(c["Hq"]):
            e = ((q[:, h] @ k[:, h // G].T) / c["D"] ** 0.5 - s["lse"][starts[n]:starts[n + 1], h, None].double()).exp()
            e[hidden] = 0
            w[:, h // G] += e.sum(0)
        weights[rows // P, :, rows % P] = w
    return {"weights": weights}


def exact(case, seed):
    if case["kind"] == "evict":
        return None  # whole numbers, and values that only move
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "weigh": _exact_weigh}[case["kind"]](s)
