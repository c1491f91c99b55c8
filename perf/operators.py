"""The performance cases of the paged-cache operators: what a serving program asks of them.

A serving program runs four calls around the draft path, over a cache kept in pages:

  plan    one step's page tables, slot maps and positions from the requests' lengths
  rope    norms of queries and keys for each head, rotation, keys and values into their slots
  window  attention over the pages with a sliding window and first tokens that stay visible
  prefix  attention of a batch whose requests share one long prefix

Sizes come from the configurations, tests and benchmark of this repository (blocks of 16, 1 to 256
requests, heads of 128) or are generic. Lengths follow a fixed low-discrepancy pattern, so that a
case's work is known without its inputs; values and the order of the pages come from the seed.
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


def _plan(name, N, block, ctx, page, window=0, sinks=0, chunk=0, ending=0):
    """block new tokens a request; of every 16 one brings a prefill chunk, of every `ending` one ends."""
    return _named(name, {"kind": "plan", "N": N, "block": block, "ctx": ctx, "page": page,
                         "window": window, "sinks": sinks, "chunk": chunk, "ending": ending})


def _rope(name, T, Hq, Hkv, D, rot, dtype="bf16", interleaved=False, page=16, norm=True):
    return _named(name, {"kind": "rope", "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot,
                         "dtype": dtype, "interleaved": interleaved, "page": page, "norm": norm})


def _window(name, N, lo, hi, ctx_lo, ctx_hi, Hq, Hkv, D, window, sinks, page, dtype="bf16",
            causal=True):
    """lo .. hi new tokens and ctx_lo .. ctx_hi tokens in the cache before them, per request."""
    return _named(name, {"kind": "window", "N": N, "lo": lo, "hi": hi, "ctx_lo": ctx_lo,
                         "ctx_hi": ctx_hi, "Hq": Hq, "Hkv": Hkv, "D": D, "window": window,
                         "sinks": sinks, "page": page, "dtype": dtype, "causal": causal})


def _prefix(name, N, lo, hi, shared, ctx_lo, ctx_hi, Hq, Hkv, D, page, dtype="bf16"):
    return _named(name, {"kind": "prefix", "N": N, "lo": lo, "hi": hi, "shared": shared,
                         "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "Hq": Hq, "Hkv": Hkv, "D": D,
                         "page": page, "dtype": dtype, "window": 0, "sinks": 0, "causal": True})


def listed():
    return [
        # one user's block of 16: nothing but latency
        _plan("plan one block", 1, 16, 2000, 16),
        # a busy server with a window: blocks, prefill chunks, ended requests, pages coming back
        _plan("plan 256 windowed", 256, 16, 16384, 16, window=4096, sinks=4, chunk=1024, ending=11),
        # one user, one token
        _rope("rope one token", 1, 32, 8, 128, 128),
        # a step full of prefill chunks, half of each head rotated, neighbouring pairs
        _rope("rope prefill fp16", 16381, 32, 8, 128, 64, dtype="fp16", interleaved=True, page=64),
        # one user, one token, a long conversation behind a window
        _window("window one token", 1, 1, 1, 32767, 32767, 32, 8, 128, 4096, 4, 16),
        # the benchmark's batch: the target checks 64 blocks of 16 drafted tokens
        _window("window 64 blocks", 64, 16, 16, 1000, 16000, 32, 8, 128, 4096, 4, 16),
        # a full server, one token each, no window: the largest read
        _window("window 256 tokens", 256, 1, 1, 100, 8100, 32, 8, 128, 0, 0, 64),
        # a prefill chunk behind a long context: matrix work
        _window("window prefill", 1, 8192, 8192, 4096, 4096, 32, 8, 128, 4096, 4, 16),
        # nothing is a round number: blocks of any length, none among them, seen from both sides
        _window("window ragged fp16", 37, 0, 33, 0, 5000, 14, 2, 64, 1000, 7, 24, dtype="fp16",
                causal=False),
        # a lightly loaded server whose requests share a system prompt, one token each
        _prefix("prefix 32 tokens", 32, 1, 1, 8192, 10, 500, 32, 8, 128, 16),
        # the benchmark's batch of blocks behind a long shared document
        _prefix("prefix 64 blocks", 64, 16, 16, 16384, 50, 1000, 32, 8, 128, 16),
        # odd: a prefix that ends inside a page, heads of 80, three query heads to a key head
        _prefix("prefix odd fp16", 11, 0, 9, 5003, 0, 700, 12, 4, 80, 24, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choices(("plan", "rope", "window", "prefix"), (2, 2, 5, 3))[0]
        page = rng.choice((8, 16, 16, 16, 24, 32, 64, 128))
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        Hkv, G = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 6, 8))
        D = rng.choice((64, 64, 80, 96, 128, 128, 128, 256))
        window, sinks = (_log(rng, 128, 4096), rng.choice((0, 1, 4, 4, 7, 64))) if rng.random() < 0.6 else (0, 0)
        if kind == "plan":
            c = _plan(None, _log(rng, 1, 256), rng.randint(1, 17), _log(rng, 100, 16384), page,
                      window, sinks, rng.choice((0, 0, _log(rng, 64, 1024))), rng.choice((0, 5, 11)))
        elif kind == "rope":
            c = _rope(None, _log(rng, 1, 16381), Hkv * G, Hkv, D,
                      16 * rng.randint(1, D // 16), dtype, rng.random() < 0.3, page, rng.random() < 0.8)
        else:
            form = rng.choice(("token", "block", "block", "ragged", "prefill"))
            N = _log(rng, 1, 256)
            lo, hi = {"token": (1, 1), "block": (16, 16), "ragged": (0, _log(rng, 2, 300)),
                      "prefill": (1, _log(rng, 200, 8192))}[form]
            if form == "prefill":
                N = max(1, N // 32)
            ctx = _log(rng, 16, 32767)
            if kind == "window":
                c = _window(None, N, lo, hi, rng.choice((0, ctx // 8, ctx)), ctx, Hkv * G, Hkv, D,
                            window, sinks, page, dtype, rng.random() < 0.8)
            else:
                tail = _log(rng, 16, 2000)
                c = _prefix(None, N, min(lo, 512), min(hi, 512), _log(rng, 500, 16384),
                            rng.choice((0, tail // 8)), tail, Hkv * G, Hkv, D, page, dtype)
        # no dearer than the largest listed cases, and a plain form that fits the card
        w = work(c)
        if w["bytes"] > 4.2e9 or w["flops"] > 5.6e11:
            continue
        if kind in ("window", "prefix"):
            new, _, total = _lengths(c)
            keys = max(total) + c.get("shared", 0)
            if max(new) * c["N"] * c["Hq"] * keys > 3.6e9 or c["N"] * keys * c["Hkv"] * D > 3.6e9:
                continue
            if sum(new) == 0:
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


def _plan_lengths(c):
    """lengths, incoming and pages (filled, returned) of every request before the step."""
    P, W, N = c["page"], c["window"], c["N"]
    first = -(-c["sinks"] // P) if W else 0
    lengths, incoming, pages = [], [], []
    for n in range(N):
        L = _spread(n, c["ctx"] // 16, c["ctx"], 0.7548776662)
        I = c["block"]
        if c["chunk"] and n % 16 == 3:
            L, I = L // 2, c["chunk"]
        if c["ending"] and n % c["ending"] == 5:
            I = -1
        end = -(-(L + n % (P + 1)) // P)  # some hold a page for tokens that were rejected
        # what the window left behind one block ago
        back = max(first, min(end, max(0, (L - 16 - W + 1) // P))) if W else 0
        lengths.append(L)
        incoming.append(I)
        pages.append((end, back))
    return lengths, incoming, pages


def _visible(p, total, c):
    """Keys that the query at position p sees."""
    hi = min(total, p + 1) if c["causal"] else total
    if not c["window"]:
        return max(0, hi)
    lo = max(0, p - c["window"] + 1)
    return max(0, hi - lo) + min(c["sinks"], lo, max(hi, 0))


def work(case):
    c = case
    if c["kind"] == "plan":
        lengths, incoming, pages = _plan_lengths(c)
        tokens = sum(max(i, 0) for i in incoming)
        fresh = sum(max(0, -(-(l + i) // c["page"]) - p[0]) for l, i, p in zip(lengths, incoming, pages) if i > 0)
        return {"bytes": c["N"] * (4 + 4 + 8 + 8 + 4 + 4) + tokens * 8 + fresh * 8 + 52, "flops": 0}
    if c["kind"] == "rope":
        heads = c["Hq"] + 2 * c["Hkv"]
        return {"bytes": c["T"] * (heads * c["D"] * 4 + c["rot"] * 4 + 8),
                "flops": c["T"] * (c["Hq"] + c["Hkv"]) * c["D"] * 7}
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
    if c["kind"] == "prefix":
        pairs += sum(new) * c["shared"]
        keys += c["shared"]
    return {"bytes": keys * c["Hkv"] * c["D"] * 4 + 2 * sum(new) * c["Hq"] * c["D"] * 2 + keys * 4 // c["page"],
            "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed, tag):
    return torch.Generator(device="cuda").manual_seed((seed * 1_000_003 + tag) & ((1 << 62) - 1))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(shape, dtype, g, scale=1.0):
    """Standard normal values, a piece at a time so that no 32-bit copy of a whole cache exists."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        part = flat[at:at + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(scale))
    return out


def _tables(counts, width, order):
    """Table [N, width] whose row n lists the next counts[n] pages of `order`, -1 after them."""
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for n, k in enumerate(counts):
        table[n, :k] = order[at:at + k]
        at += k
    return table


def _prepare_plan(c, seed):
    g, P = _generator(seed, 1), c["page"]
    lengths, incoming, pages = _plan_lengths(c)
    held = sum(p[0] for p in pages)
    most = max(l + max(i, 0) for l, i in zip(lengths, incoming))
    fresh = sum(max(0, -(-(l + i) // P) - p[0]) for l, i, p in zip(lengths, incoming, pages) if i > 0)
    total = held + fresh + SPARE
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = _tables([p[0] for p in pages], -(-most // P) + 2, order)
    free = order[held:]
    # the queue of free pages has gone round an arbitrary number of times
    head = int(torch.randint(0, 5 * total, (1,), generator=g, device="cuda"))
    queue = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    queue[(head + torch.arange(free.numel(), device="cuda")) % total] = free
    return {"c": c, "lengths": _i32(lengths), "incoming": _i32(incoming), "pages": _i32(pages),
            "table": table, "queue": queue,
            "cursor": torch.tensor([head, head + free.numel(), 0], device="cuda"),
            "tokens": sum(max(i, 0) for i in incoming)}


def _prepare_rope(c, seed):
    T, Hq, Hkv, D, rot, P = (c[k] for k in ("T", "Hq", "Hkv", "D", "rot", "page"))
    g, dtype = _generator(seed, 2), DTYPE[c["dtype"]]
    # one projection's output, of which queries, keys and values are views
    qkv = _normal((T, (Hq + 2 * Hkv) * D), dtype, g, 1.5)
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
         "k_cache": _normal((pages, P, Hkv, D), dtype, g), "v_cache": _normal((pages, P, Hkv, D), dtype, g),
         "q_weight": None, "k_weight": None, "out": torch.empty(T, Hq, D, dtype=dtype, device="cuda")}
    if c["norm"]:
        for name in ("q_weight", "k_weight"):
            s[name] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    return s


def _prepare_attention(c, seed):
    N, Hq, Hkv, D, P = (c[k] for k in ("N", "Hq", "Hkv", "D", "page"))
    g, dtype = _generator(seed, 3), DTYPE[c["dtype"]]
    new, _, total = _lengths(c)
    counts = [-(-t // P) for t in total]
    shared = -(-c.get("shared", 0) // P)
    pages = sum(counts) + shared + SPARE
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    starts = [0]
    for t in new:
        starts.append(starts[-1] + t)
    T = starts[-1]
    # heads of different sharpness: scores of a standard deviation from 0.5 to 4
    q = _normal((T, Hq, D), dtype, g)
    q *= (0.5 * 2.0 ** (torch.arange(Hq, device="cuda") % 4)).to(dtype)[None, :, None]
    s = {"c": c, "q": q, "k_cache": _normal((pages, P, Hkv, D), dtype, g),
         "v_cache": _normal((pages, P, Hkv, D), dtype, g),
         "table": _tables(counts, max(counts) + 1, order[shared:]), "starts": _i32(starts),
         "totals": _i32(total), "out": torch.empty_like(q),
         "most_tokens": max(new), "most_keys": max(total), "workspace": None}
    if c["kind"] == "prefix":
        s["shared_table"] = order[:shared].contiguous()
    return s


def prepare(case, seed):
    return {"plan": _prepare_plan, "rope": _prepare_rope, "window": _prepare_attention,
            "prefix": _prepare_attention}[case["kind"]](case, seed)


# ---- one pass --------------------------------------------------------------------------------------

def _plain_plan(s):
    c, P, M, C = s["c"], s["c"]["page"], s["table"].shape[1], s["queue"].numel()
    W, first = c["window"], (-(-c["sinks"] // c["page"]) if c["window"] else 0)
    L, I = s["lengths"].long(), s["incoming"].long()
    end, back = s["pages"].long().unbind(1)
    head, tail = s["cursor"][0], s["cursor"][1]
    ended = I < 0
    fresh = torch.where(ended, 0, I)
    total = torch.where(ended, 0, L + fresh)
    take = torch.where(ended, 0, ((total + P - 1) // P).clamp(max=M) - end).clamp(min=0)
    since = torch.where(back > first, back, first)
    upto = torch.minimum(end, torch.div(L - W + 1, P, rounding_mode="floor").clamp(min=0)) if W else torch.zeros_like(end)
    kept = end.clamp(max=first)  # pages of the first tokens, given back when the request ends
    give = torch.where(ended, kept + (end - since).clamp(min=0), (upto - since).clamp(min=0))
    before, gave, at = take.cumsum(0) - take, give.cumsum(0) - give, fresh.cumsum(0)
    free = tail - head
    granted = torch.minimum(take, (free - before).clamp(min=0))
    pages = torch.stack((torch.where(ended, 0, end + granted), torch.where(ended, 0, since + give)), 1)
    cursor = torch.stack((head + torch.minimum(free, take.sum()), tail + give.sum(),
                          (take.sum() - free).clamp(min=0)))
    starts = torch.cat((at.new_zeros(1), at)).clamp(max=s["tokens"])
    # new pages into the table
    n = torch.repeat_interleave(take)
    i = torch.arange(n.numel(), device=n.device) - before[n]
    g = before[n] + i
    table = s["table"]
    table[n, end[n] + i] = torch.where(g < free, s["queue"][(head + g) % C], -1)
    # returned pages to the end of the queue
    n = torch.repeat_interleave(give)
    r = torch.arange(n.numel(), device=n.device) - gave[n]
    e = torch.where(ended[n], torch.where(r < kept[n], r, since[n] + r - kept[n]), since[n] + r)
    s["queue"][(tail + gave[n] + r) % C] = table[n, e]
    # slots and positions
    n = torch.repeat_interleave(fresh)
    position = L[n] + torch.arange(n.numel(), device=n.device) - (at - fresh)[n]
    e = position // P
    page = torch.where(e < pages[n, 0], table[n, e.clamp(max=M - 1)].long(), -1)
    slots = torch.where(page >= 0, page * P + position % P, -1)
    i32 = torch.int32
    return {"table": table, "queue": s["queue"], "pages": pages.to(i32), "cursor": cursor, "starts": starts.to(i32),
            "totals": total.to(i32), "slots": slots.to(i32), "positions": position.to(i32)}


def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), rest), -1)
    a, b = r[..., :rot // 2], r[..., rot // 2:]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)


def _plain_rope(s):
    c, dtype = s["c"], s["q"].dtype
    cos, sin = s["cos_sin"][s["positions"].long()][:, None].chunk(2, -1)
    made = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
        made.append(_rotated(x, cos, sin, c["interleaved"]).to(dtype))
    live = s["slots"] >= 0
    at = s["slots"][live].long()
    s["k_cache"].view(-1, c["Hkv"], c["D"])[at] = made[1][live]
    s["v_cache"].view(-1, c["Hkv"], c["D"])[at] = s["v"][live]
    return {"q": made[0], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    c, q, P = s["c"], s["q"], s["c"]["page"]
    N, Hkv, D, G, W = c["N"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"], c["window"]
    dev, most, keys = q.device, s["most_tokens"], s["most_keys"]
    starts, total = s["starts"].long(), s["totals"].long()
    new = starts[1:] - starts[:-1]
    # queries padded to [N, Hkv, most * G, D], keys and values gathered to [N, Hkv, keys, D]
    t = torch.arange(most, device=dev)
    live = t < new[:, None]
    at = torch.where(live, starts[:-1, None] + t, 0)
    x = q[at].float().view(N, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(N, Hkv, most * G, D)
    j = torch.arange(keys, device=dev)
    page = s["table"].long()[:, j // P]
    held = (page >= 0) & (j < total[:, None])
    slot = torch.where(held, page * P + j % P, 0)
    k, v = (s[n].view(-1, Hkv, D)[slot].permute(0, 2, 1, 3).float() for n in ("k_cache", "v_cache"))
    p = (total - new)[:, None] + t
    seen = held[:, None, :].expand(N, most, keys)
    if c["causal"]:
        seen = seen & (j <= p[:, :, None])
    if W:
        seen = seen & ((j > p[:, :, None] - W) | (j < c["sinks"]))
    seen = seen.repeat_interleave(G, 1)[:, None]
    scores = torch.matmul(x, k.transpose(2, 3)).mul_(1 / math.sqrt(D)).masked_fill_(~seen, -math.inf)
    if c["kind"] == "prefix":
        j = torch.arange(c["shared"], device=dev)
        slot = s["shared_table"].long()[j // P] * P + j % P
        k0, v0 = (s[n].view(-1, Hkv, D)[slot].permute(1, 0, 2).float() for n in ("k_cache", "v_cache"))
        first = torch.matmul(x, k0.transpose(1, 2)).mul_(1 / math.sqrt(D))
        m = torch.maximum(first.amax(-1, keepdim=True), scores.amax(-1, keepdim=True))
        first, scores = first.sub_(m).exp_(), scores.sub_(m).exp_()
        o = torch.matmul(first, v0) + torch.matmul(scores, v)
        o = o / (first.sum(-1, keepdim=True) + scores.sum(-1, keepdim=True))
    else:
        m = scores.amax(-1, keepdim=True)
        scores = scores.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
        z = scores.sum(-1, keepdim=True)
        o = torch.matmul(scores, v) / torch.where(z == 0, 1.0, z)
    o = o.view(N, Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(N, most, Hkv * G, D)
    return o[live].to(q.dtype)


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"plan": _plain_plan, "rope": _plain_rope, "window": _plain_attention,
                "prefix": _plain_attention}[c["kind"]](s)
    import paper_2608_20530_amd as L
    if c["kind"] == "plan":
        p = L.page_plan(s["lengths"], s["incoming"], s["pages"], s["table"], s["queue"], s["cursor"],
                        page_size=c["page"], tokens=s["tokens"], window=c["window"], sinks=c["sinks"])
        return {"table": s["table"], "queue": s["queue"], "pages": p.pages, "cursor": p.cursor, "starts": p.starts,
                "totals": p.totals, "slots": p.slots, "positions": p.positions}
    if c["kind"] == "rope":
        q = L.qk_norm_rope(s["q"], s["k"], s["v"], s["slots"], s["positions"], s["cos_sin"],
                           s["k_cache"], s["v_cache"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                           eps=EPS, interleaved=c["interleaved"], out=s["out"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    bounds = {"max_tokens": s["most_tokens"], "max_length": s["most_keys"]}
    if c["kind"] == "prefix":
        if s["workspace"] is None:  # made by the first pass and kept
            s["workspace"] = L.prefix_attention_workspace(s["q"], s["k_cache"], s["table"], c["shared"],
                                                          **bounds)
        return L.prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["shared_table"], c["shared"],
                                  s["table"], s["starts"], s["totals"], out=s["out"],
                                  workspace=s["workspace"], **bounds)
    mask = {"window": c["window"], "sinks": c["sinks"], "causal": c["causal"]}
    if s["workspace"] is None:
        s["workspace"] = L.window_attention_workspace(s["q"], s["k_cache"], s["table"], **mask, **bounds)
    return L.window_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["totals"],
                              out=s["out"], workspace=s["workspace"], **mask, **bounds)


# ---- the definition in 64 bits ---------------------------------------------------------------------

def _exact_rope(s):
    """Each pair as a complex number, turned by its angle's; a head is normed by its 2-norm."""
    c = s["c"]
    half = c["rot"] // 2
    table = s["cos_sin"].double()
    turn = torch.complex(table[:, :half], table[:, half:])[s["positions"].long()][:, None]
    out = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.double()
        if w is not None:
            norm = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
            x = x / (norm * norm / c["D"] + EPS).sqrt() * w.double()
        x = x.clone()
        pairs = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else \
            (slice(0, half), slice(half, c["rot"]))
        z = torch.complex(x[..., pairs[0]], x[..., pairs[1]]) * turn
        x[..., pairs[0]], x[..., pairs[1]] = z.real, z.imag
        out.append(x)
    k_cache, v_cache = (s[n].double().flatten(0, 1) for n in ("k_cache", "v_cache"))
    live = (s["slots"] >= 0).nonzero().flatten()
    k_cache.index_copy_(0, s["slots"][live].long(), out[1][live])
    v_cache.index_copy_(0, s["slots"][live].long(), s["v"].double()[live])
    shape = s["k_cache"].shape
    return {"q": out[0], "k_cache": k_cache.view(shape), "v_cache": v_cache.view(shape)}


def _exact_attention(s):
    """Request by request and head by head, the keys of a row named one by one in a list of bounds."""
    c, P = s["c"], s["c"]["page"]
    G, D, W = c["Hq"] // c["Hkv"], c["D"], c["window"]
    starts, totals = s["starts"].tolist(), s["totals"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    flat = {n: s[n].flatten(0, 1) for n in ("k_cache", "v_cache")}
    shared = c.get("shared", 0)

    def rows_of(table, length):
        at = torch.arange(length, device="cuda")
        return table.long()[at // P] * P + at % P

    common = rows_of(s["shared_table"], shared) if shared else None
    for n, total in enumerate(totals):
        new = starts[n + 1] - starts[n]
        if not new:
            continue
        rows = rows_of(s["table"][n], total)
        if shared:
            rows = torch.cat((common, rows))
        k, v = (flat[m][rows].double() for m in ("k_cache", "v_cache"))  # [keys, Hkv, D]
        q = s["q"][starts[n]:starts[n + 1]].double()
        at = torch.arange(total + shared, device="cuda")[None] - shared
        step = max(1, (1 << 27) // (total + shared))
        for b in range(0, new, step):
            p = torch.arange(total - new + b, total - new + min(b + step, new), device="cuda")[:, None]
            hidden = (at > p) if c["causal"] else torch.zeros_like(at > p)
            if W:
                hidden = hidden | ((at <= p - W) & (at >= c["sinks"]))
            for h in range(c["Hq"]):
                z = (q[b:b + step, h] @ k[:, h // G].T) / D ** 0.5
                z[hidden] = -math.inf
                e = (z - torch.logsumexp(z, 1, keepdim=True)).exp()
                out[starts[n] + b:starts[n] + b + p.shape[0], h] = torch.nan_to_num(e) @ v[:, h // G]
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None  # whole numbers
    s = prepare(case, seed)
    return _exact_rope(s) if c["kind"] == "rope" else _exact_attention(s)
