"""GPU tests of the 4-bit cache's calls against the plain 64-bit definitions (oracle/cache4.py).

Tolerances, from the roundings that the calls make (u = 2^-8 for bf16, 2^-11 for fp16: half a unit in the last
place, relative to the value; codes are exact in bf16):
  codes, scales, whole numbers, what moves   equal
  attention   u |o| for the output; 2^-8 sum p|v| for the probabilities (bf16, whatever the type), 2^-16 with fp16 (two
              terms); for the fp32 scores an error e of at most 2^-24 ((d + 2) S + 4 |s|), S = scale sum |q_i k_i|
              >= |s|, which moves the result by at most 2 e sum p|v|; n 2^-23 sum p|v| for fp32 sums over n keys
  lse         e; n 2^-24 for the sum, 2^-22 for the powers; 2^-22 (|lse| + S + 10) for the logarithm's parts
  weights     each term exp(s - lse): e, 2^-22 for the power and 2^-22 |lse| for its argument's second part, relative, all
              below 2^-24 (d + 8) (1 + S + |lse|); (terms + 4) 2^-24 of the result for the sum
"""
import numpy as np
import pytest
import torch

import oracle.cache4 as ref
import oracle.paged

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
U = {BF: 2.0 ** -8, HF: 2.0 ** -11}
P_U = {BF: 2.0 ** -8, HF: 2.0 ** -16}
TINY = {BF: 0.0, HF: 2.0 ** -25}


def f64(t):
    return t.detach().double().cpu().numpy()


def host(t):
    return t.detach().cpu().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def make_cache(lib, pages, page, heads, d, layout="phd", g=None, scale=1.0):
    """A cache of normal values in one of four layouts; untouched parts are whatever the seed says."""
    g = g or torch.Generator().manual_seed(0)
    codes = [torch.randint(0, 256, (pages, page, heads, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.randint(124, 128, (pages, page, heads, d // 32), generator=g, dtype=torch.uint8) for _ in range(2)]

    def laid(x):
        if layout == "hpd":  # heads outside a page's tokens
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        if layout == "wide":  # tokens with room behind them: strides that are no power of two
            room = torch.zeros(pages, page, heads + 1, x.shape[3], dtype=torch.uint8)
            room[:, :, :heads] = x
            return room.cuda()[:, :, :heads]
        return x.cuda()

    if layout == "kv":  # keys and values of a page side by side
        k, v = torch.stack(codes, 1).cuda().unbind(1)
        ks, vs = torch.stack(scales, 1).cuda().unbind(1)
        return lib.Cache4(k, ks, v, vs)
    k, v = map(laid, codes)
    ks, vs = map(laid, scales)
    return lib.Cache4(k, ks, v, vs)


def values(cache):
    return ref.values(host(cache.k), host(cache.k_scales)), ref.values(host(cache.v), host(cache.v_scales))


# ---- the write --------------------------------------------------------------------------------------

def rope_inputs(lib, T, Hq, Hkv, d, rot, dtype, norm=True, page=16, layout="phd", seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    qkv = r(T, (Hq + 2 * Hkv) * d).to(dtype).cuda()
    q, k, v = (qkv[:, a * d:b * d].view(T, b - a, d) for a, b in
               ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    pages = T // page * 2 + 3
    cache = make_cache(lib, pages, page, Hkv, d, layout, g)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    slots[(T + 1) // 2:(T + 1) // 2 + 1] = -1
    positions = torch.randint(0, 5000, (T,), generator=g).to(torch.int32)
    if T > 3:
        positions[3], slots[2] = -1, pages * page  # no token; a slot that is not there
        positions[1] = 5000                        # past the table
    ang = torch.rand(5000, max(rot // 2, 1), generator=g, dtype=torch.float64)[:, :rot // 2] * 6.3
    cs = torch.cat((ang.cos(), ang.sin()), 1).float().cuda() if rot else None
    w = [1 + 0.2 * r(d).cuda() if norm else None for _ in range(2)]
    return q, k, v, slots.cuda(), positions.cuda(), cs, cache, w


ROPE_CASES = [
    # T, Hq, Hkv, d, rot, dtype, interleaved, norm, page, layout
    (1, 32, 8, 128, 128, BF, False, True, 16, "phd"),
    (1, 1, 1, 32, 16, HF, True, True, 1, "phd"),
    (17, 8, 8, 64, 64, BF, False, True, 16, "hpd"),
    (33, 12, 4, 96, 96, HF, False, True, 24, "kv"),
    (20, 6, 2, 96, 32, BF, False, True, 16, "wide"),
    (20, 5, 1, 256, 256, BF, False, False, 8, "phd"),
    (9, 14, 2, 224, 112, HF, True, True, 16, "kv"),
    (7, 3, 3, 32, 16, BF, True, False, 16, "hpd"),
    (10, 4, 2, 128, 0, HF, False, True, 16, "phd"),
    (150, 32, 8, 128, 128, BF, False, True, 16, "kv"),
    (301, 5, 3, 160, 64, HF, True, True, 16, "wide"),
    (2101, 4, 1, 128, 128, BF, False, True, 16, "hpd"),
]


def check_write(q, k, v, slots, positions, cs, cache, w, out, before, dtype, rot, inter, eps=1e-5):
    """Codes and scales equal to the definition's, other places as they were; q within its rounding."""
    pos, sl = host(positions), host(slots)
    live = (pos >= 0) & (pos < 5000) if rot else pos >= 0
    at = np.where(live, pos, 0)
    table = f64(cs) if rot else np.zeros((5001, 0))
    c, s = table[at, :rot // 2], table[at, rot // 2:]
    eps = float(np.float32(eps))
    want_q, want_k = [oracle.paged.norm_rope(f64(x), f64(y) if y is not None else None, c, s, eps, inter)
                      for x, y in ((q, w[0]), (k, w[1]))]
    want_q[~live] = 0
    tol = U[dtype] * np.abs(want_q) + 4e-6 * np.abs(want_q).max(-1, keepdims=True) + TINY[dtype]
    assert (np.abs(f64(out) - want_q) <= tol).all()
    P, pages = cache.k.shape[1], cache.k.shape[0]
    stored = live & (sl >= 0) & (sl < pages * P)
    want = [x.copy() for x in before]
    for i, x in ((0, want_k), (2, f64(v))):
        codes, scales = ref.quantise(x[stored])
        want[i].reshape(pages * P, *want[i].shape[2:])[sl[stored]] = codes
        want[i + 1].reshape(pages * P, *want[i + 1].shape[2:])[sl[stored]] = scales
    for name, a, b in zip(cache._fields, cache, want):
        bad = np.argwhere(host(a) != b)
        assert not len(bad), f"{name}: {len(bad)} differ, first {bad[0]}: {host(a)[tuple(bad[0])]} {b[tuple(bad[0])]}"


@pytest.mark.parametrize("T,Hq,Hkv,d,rot,dtype,inter,norm,page,layout", ROPE_CASES)
def test_qk_norm_rope4(lib, T, Hq, Hkv, d, rot, dtype, inter, norm, page, layout):
    q, k, v, slots, positions, cs, cache, w = rope_inputs(lib, T, Hq, Hkv, d, rot, dtype, norm, page, layout)
    before = [np.ascontiguousarray(host(x)) for x in cache]
    out = lib.qk_norm_rope4(q, k, v, slots, positions, cs, cache, q_weight=w[0], k_weight=w[1], eps=1e-5,
                            interleaved=inter)
    torch.cuda.synchronize()
    check_write(q, k, v, slots, positions, cs, cache, w, out, before, dtype, rot, inter)
    again = lib.qk_norm_rope(q, *(x for x in (k, v)), slots, positions, cs,
                             *(torch.zeros(*cache.k.shape[:3], d, dtype=dtype, device="cuda") for _ in range(2)),
                             q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=inter)
    assert torch.equal(out, again), "queries are those of the 16-bit cache's call"


@pytest.mark.parametrize("dtype", [BF, HF])
def test_codes_at_their_borders(lib, dtype):
    """Ties, signs, zeros and ends of the range, as they are (no norm, no rotation), in every lane."""
    d, T = 64, 64
    steps = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    top = {BF: 2.0 ** 127, HF: 2.0 ** 14}[dtype]
    least = {BF: 2.0 ** -133, HF: 2.0 ** -24}[dtype]
    x = torch.zeros(T, 2, d)
    for t in range(T):
        x[t, 0, :32] = torch.cat((steps, -steps)).roll(t) * 2.0 ** (t % 20 - 10)
        x[t, 0, 32:] = torch.cat((steps, -steps)).roll(3 * t) * 2.0 ** -12
        x[t, 1, t % 64] = (top * 1.75, top * 1.9, -top, least, -least * 3, 7.03125, 7.0, -0.0)[t % 8]
    x = x.to(dtype).cuda()
    cache = make_cache(lib, 8, 8, 2, d)
    before = [np.ascontiguousarray(host(y)) for y in cache]
    slots, positions = i32(list(range(T))), i32([0] * T)
    out = lib.qk_norm_rope4(x, x, x, slots, positions, None, cache)
    torch.cuda.synchronize()
    check_write(x, x, x, slots, positions, None, cache, (None, None), out, before, dtype, 0, False)


def test_keys_that_fp32_does_not_decide(lib):
    """Rotations that cancel or land on the borders of codes and scales: the codes are those of 64 bits."""
    d, T = 64, 96
    g = torch.Generator().manual_seed(5)
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    a = steps[torch.randint(0, 8, (T, 1, 32), generator=g)]
    b = a * torch.randint(-1, 2, (T, 1, 32), generator=g)
    k = torch.cat((a, b), 2).to(BF).cuda()
    # angles whose sine and cosine are equal, or nearly: a c - b s is 0, or 2^-24 of a
    c = torch.full((T, 32), 0.70710678) + torch.randint(-1, 2, (T, 32), generator=g) * 2.0 ** -24
    cs = torch.cat((c, torch.full((T, 32), 0.70710678)), 1)
    cs[: T // 3, :32], cs[: T // 3, 32:] = 1.0, 2.0 ** -26  # a little beside a border
    cs[T // 3: T // 2, 32:] = -(2.0 ** -26)
    cs[T // 3: T // 2, :32] = 1.0
    w = torch.ones(d).cuda()
    for weight in (None, w):
        cache = make_cache(lib, 12, 8, 1, d)
        before = [np.ascontiguousarray(host(y)) for y in cache]
        slots, positions = i32(list(range(T))), i32(list(range(T)))
        table = torch.zeros(5000, d)
        table[:T] = cs
        out = lib.qk_norm_rope4(k, k, k, slots, positions, table.cuda(), cache, k_weight=weight, eps=0.0)
        torch.cuda.synchronize()
        check_write(k, k, k, slots, positions, table, cache, (None, weight), out, before, BF, d, False, eps=0.0)


def test_infinities_and_nan_make_nan_blocks(lib):
    x = torch.randn(4, 2, 64, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    x[0, 0, 5], x[1, 1, 40], x[2, 0, 63] = float("inf"), float("nan"), -float("inf")
    cache = lib.cache4(2, 2, 2, 64)
    lib.qk_norm_rope4(x, x, x, i32([0, 1, 2, 3]), i32([0] * 4), None, cache)
    torch.cuda.synchronize()
    for codes, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        want = np.zeros((4, 2, 2), bool)
        want[0, 0, 0] = want[1, 1, 1] = want[2, 0, 1] = True
        assert np.array_equal(host(scales).reshape(4, 2, 2) == 255, want)
        c, s = ref.quantise(f64(x))
        assert np.array_equal(host(scales).reshape(4, 2, 2), s)
        assert np.array_equal(host(codes).reshape(4, 2, 32), c)


def test_qk_norm_rope4_in_place_and_empty(lib):
    q, k, v, slots, positions, cs, cache, w = rope_inputs(lib, 40, 8, 2, 128, 128, BF, seed=3)
    q = q.contiguous()
    want = lib.qk_norm_rope4(q, k, v, slots, positions, cs, cache, q_weight=w[0], k_weight=w[1])
    got = lib.qk_norm_rope4(q, k, v, slots, positions, cs, cache, q_weight=w[0], k_weight=w[1], out=q)
    torch.cuda.synchronize()
    assert got is q and torch.equal(got, want)
    kept = cache.k.clone()
    out = lib.qk_norm_rope4(q[:0], k[:0], v[:0], slots[:0], positions[:0], cs, cache)
    torch.cuda.synchronize()
    assert out.shape == (0, 8, 128) and torch.equal(cache.k, kept)


# ---- attention --------------------------------------------------------------------------------------

def attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype, layout="phd", seed=0, pad_rows=0):
    g = torch.Generator().manual_seed(seed)
    totals = [a + b for a, b in zip(new, ctx)]
    counts = [-(-t // page) for t in totals]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(new), max(max(counts), 1) + 1), -1, dtype=torch.int32)
    at = 0
    for n, c in enumerate(counts):
        table[n, :c] = order[at:at + c]
        at += c
    starts = np.concatenate(([0], np.cumsum(new))).tolist()
    sharp = (0.25 * 2.0 ** (torch.arange(Hq) % 3))[None, :, None]
    q = (torch.randn(starts[-1] + pad_rows, Hq, d, generator=g) * sharp).to(dtype).cuda()
    return dict(q=q, cache=make_cache(lib, pages, page, Hkv, d, layout, g), table=table.cuda(), starts=i32(starts),
                totals=i32(totals))


def attend(lib, x, **kw):
    lse = torch.full(x["q"].shape[:2], 77.0, device="cuda")
    out = lib.window_attention4(x["q"], x["cache"], x["table"], x["starts"], x["totals"], lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


def wanted(x, **mask):
    return ref.attention(f64(x["q"]), *values(x["cache"]), host(x["table"]), host(x["starts"]), host(x["totals"]),
                         **mask)


def check_attention(x, got, want):
    out, lse = got
    exact, absolute, sizes, count, exact_lse = want
    dtype, d = x["q"].dtype, x["q"].shape[2]
    e = 2.0 ** -24 * ((d + 2) * sizes + 4 * sizes)
    tol = U[dtype] * np.abs(exact) + (P_U[dtype] + 2 * e + count[:, None] * 2.0 ** -23)[..., None] * absolute + TINY[dtype]
    bad = ~(np.abs(f64(out) - exact) <= tol)
    assert not bad.any(), (f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: "
                           f"{f64(out)[bad][0]!r} for {exact[bad][0]!r}, bound {tol[bad][0]!r}")
    used = int(x["starts"][-1])
    lse, exact_lse = f64(lse)[:used], exact_lse[:used]
    empty = exact_lse == -np.inf
    assert np.array_equal(lse == -np.inf, empty)
    near = np.where(empty, 0, exact_lse)
    tol = (e + count[:, None] * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(sizes) + 10))[:used] + 2.0 ** -22 * np.abs(near)
    bad = ~(np.abs(np.where(empty, 0, lse) - near) <= tol)
    assert not bad.any(), f"lse: {lse[bad][0]!r} for {near[bad][0]!r}, bound {tol[bad][0]!r}"


ATTENTION_CASES = [
    # new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype
    ([1], [0], 1, 1, 64, 16, 0, 0, True, BF),
    ([1], [700], 32, 8, 128, 16, 0, 0, True, BF),
    ([1], [700], 32, 8, 128, 16, 100, 4, True, HF),
    ([1, 1, 1], [0, 31, 32], 4, 2, 64, 8, 0, 0, True, HF),
    ([1, 1, 1, 1], [63, 64, 65, 300], 8, 8, 128, 1, 64, 1, True, BF),
    ([16, 16], [100, 333], 32, 8, 128, 16, 0, 0, True, BF),
    ([16, 16], [100, 333], 32, 8, 128, 16, 50, 7, True, HF),
    ([16], [400], 8, 2, 64, 16, 33, 64, False, BF),
    ([16, 3, 0, 1], [0, 5, 77, 260], 7, 1, 64, 24, 0, 0, False, HF),
    ([0, 33, 1, 17], [9, 200, 0, 64], 14, 2, 64, 24, 90, 7, False, HF),
    ([150], [0], 4, 1, 128, 16, 0, 0, True, BF),
    ([150, 70], [33, 500], 4, 1, 128, 32, 40, 3, True, BF),
    ([65], [70], 2, 2, 96, 24, 0, 0, True, HF),
    ([40, 5], [70, 300], 6, 2, 96, 128, 64, 16, True, BF),
    ([1, 2], [500, 40], 16, 2, 256, 16, 0, 0, True, BF),
    ([16, 7], [300, 90], 8, 2, 256, 16, 60, 4, True, HF),
    ([50], [90], 4, 1, 256, 16, 0, 0, True, BF),
    ([3], [20], 6, 2, 32, 4, 0, 0, True, HF),
    ([3, 20], [40, 60], 5, 1, 224, 16, 30, 2, True, BF),
    ([7], [90], 4, 2, 160, 5, 0, 0, True, HF),
    ([1], [2000], 16, 1, 64, 16, 1, 0, True, BF),       # a window of the query alone
    ([2, 9], [50, 50], 64, 1, 64, 16, 0, 0, True, BF),  # 64 query heads to a key head
    ([1] * 70, list(range(70)), 4, 2, 64, 16, 0, 0, True, BF),
    ([1, 90] * 20, list(range(40)), 2, 1, 64, 16, 33, 2, True, HF),
    ([4, 8], [900, 40], 8, 2, 128, 48, 200, 40, True, BF),
    ([8, 3], [300, 70], 8, 2, 128, 24, 0, 0, True, BF),  # pages and widths that go by way of registers
    ([16, 1], [200, 41], 8, 2, 96, 16, 0, 0, True, HF),
    ([60, 25], [100, 300], 8, 2, 128, 24, 77, 5, False, HF),
    ([90], [150], 4, 2, 96, 32, 0, 0, True, BF),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,window,sinks,causal,dtype", ATTENTION_CASES)
def test_window_attention4(lib, new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype):
    print("attention", new[:4], ctx[:4], Hq, Hkv, d, page, window, sinks, flush=True)
    x = attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype)
    mask = dict(window=window, sinks=sinks, causal=causal)
    got = attend(lib, x, **mask, max_tokens=max(new), max_length=max(a + b for a, b in zip(new, ctx)))
    check_attention(x, got, wanted(x, **mask))
    again = attend(lib, x, **mask, max_tokens=max(new), max_length=max(a + b for a, b in zip(new, ctx)))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("layout,page,d", [("hpd", 16, 128), ("kv", 16, 64), ("wide", 32, 128), ("wide", 8, 96), ("hpd", 3, 256),
                                           ("wide", 16, 160)])
def test_cache_layouts(lib, layout, page, d):
    x = attention_inputs(lib, [5, 16, 1], [100, 0, 37], 8, 2, d, page, BF, layout)
    check_attention(x, attend(lib, x), wanted(x))


def test_views_of_queries_and_bounds_that_are_loose(lib):
    x = attention_inputs(lib, [3, 9], [70, 20], 8, 2, 128, 16, BF)
    want = wanted(x)
    room = torch.zeros(12, 12, 128, dtype=BF, device="cuda")
    room[:, 2:10] = x["q"]
    x["q"] = room[:, 2:10]
    check_attention(x, attend(lib, x), want)
    check_attention(x, attend(lib, x, max_tokens=4000, max_length=1 << 20), want)


@pytest.mark.parametrize("d,causal", [(64, True), (128, False), (256, True)])
def test_pages_that_are_not_there(lib, d, causal):
    x = attention_inputs(lib, [4, 16], [90, 40], 4, 2, d, 16, BF)
    x["table"][0, 2], x["table"][1, 0], x["table"][1, 3] = -1, 10 ** 6, -5
    check_attention(x, attend(lib, x, causal=causal), wanted(x, causal=causal))


def test_rows_that_see_nothing_are_zeros(lib):
    x = attention_inputs(lib, [2, 3], [0, 40], 4, 2, 64, 16, BF, pad_rows=5)
    x["table"][0] = -1
    x["q"][5:] = float("nan")
    out, lse = attend(lib, x)
    assert torch.equal(out[:2], torch.zeros_like(out[:2])) and (lse[:2] == -float("inf")).all()
    want = wanted(dict(x, q=torch.nan_to_num(x["q"])))
    check_attention(dict(x, q=x["q"][:5]), (out[:5], lse[:5]), tuple(w[:5] for w in want))


@pytest.mark.parametrize("new,d,page,window", [([16], 64, 16, 0), ([40], 128, 24, 0), ([9], 256, 16, 0), ([3], 96, 16, 0),
                                               ([90], 128, 16, 30)])
def test_nan_blocks_reach_only_rows_that_see_them(lib, new, d, page, window):
    """NaN blocks of values and keys at places that only some rows see, and past the end: rows that do not see them are as
    without them; a value's block makes its 32 elements NaN, a key the whole row."""
    T, ctx, G = new[0], 50, 4
    x = attention_inputs(lib, new, [ctx], 2 * G, 2, d, page, BF)
    clean = attend(lib, x, window=window)
    c, row = x["cache"], host(x["table"])[0]
    total, blocks = T + ctx, d // 32
    value_at, key_at = ctx + T // 2, ctx + T - 1  # a value's second block (or only one), the last query's own key
    b = min(1, blocks - 1)
    c.v_scales[row[value_at // page], value_at % page, 1, b] = 255
    c.k_scales[row[key_at // page], key_at % page, 0, 0] = 255
    for j in range(total, -(-total // page) * page):  # behind the end of the last page
        c.v_scales[row[j // page], j % page] = 255
        c.k_scales[row[j // page], j % page] = 255
    if window:  # nobody's window reaches the first keys
        c.v_scales[row[0], 0] = 255
    out, lse = attend(lib, x, window=window)
    nan = torch.zeros_like(out, dtype=torch.bool)
    nan[T // 2:T // 2 + window if window else T, G:, 32 * b:32 * b + 32] = True  # the rows whose window has it
    nan[T - 1, :G] = True
    same = torch.equal(out.isnan(), nan), torch.equal(out[~nan], clean[0][~nan])
    assert same == (True, True)
    gone = torch.zeros_like(lse, dtype=torch.bool)
    gone[T - 1, :G] = True
    same = torch.equal(lse.isnan(), gone), torch.equal(lse[~gone], clean[1][~gone])
    assert same == (True, True)


def test_lse_is_optional_and_changes_nothing(lib):
    for new, ctx in (([1], [3000]), ([16, 16], [100, 200])):
        x = attention_inputs(lib, new, ctx, 8, 2, 128, 16, BF)
        want, _ = attend(lib, x)
        got = lib.window_attention4(x["q"], x["cache"], x["table"], x["starts"], x["totals"])
        torch.cuda.synchronize()
        assert torch.equal(got, want)


# ---- accumulated weights ------------------------------------------------------------------------------

def check_weights(got, want, before):
    exact, size, terms = want
    d_bound = 2.0 ** -24 * (256 + 8)
    tol = d_bound * size + (terms + 4) * 2.0 ** -24 * np.abs(exact)
    bad = ~(np.abs(f64(got) - exact) <= tol)
    assert not bad.any(), (f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {f64(got)[bad][0]!r} for "
                           f"{exact[bad][0]!r}, bound {tol[bad][0]!r}, before {f64(before)[bad][0]!r}")


WEIGHT_CASES = [
    # new, ctx, Hq, Hkv, d, page, causal, decay, dtype
    ([1], [0], 1, 1, 64, 16, True, 1.0, BF),
    ([1], [300], 32, 8, 128, 16, True, 0.5, BF),
    ([1, 1, 1], [0, 31, 32], 4, 2, 64, 8, True, 0.9, HF),
    ([4, 2, 0, 1], [100, 3, 50, 64], 4, 1, 96, 24, True, 1.0, BF),
    ([4, 3], [40, 90], 8, 2, 128, 16, False, 0.25, HF),
    ([16, 16], [100, 33], 16, 4, 128, 16, True, 0.98, BF),
    ([40, 0, 7], [0, 20, 130], 7, 1, 64, 1, True, 1.0, HF),
    ([33], [70], 4, 2, 256, 16, False, 0.5, BF),
    ([9, 20], [90, 5], 6, 2, 224, 32, True, 0.0, HF),
    ([5], [200], 64, 1, 32, 16, True, 1.0, BF),
    ([2], [30], 3, 3, 256, 5, True, 0.7, BF),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,causal,decay,dtype", WEIGHT_CASES)
def test_key_weights(lib, new, ctx, Hq, Hkv, d, page, causal, decay, dtype):
    print("weights", new[:4], ctx[:4], Hq, Hkv, d, page, causal, flush=True)
    x = attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype)
    _, lse = attend(lib, x, causal=causal)
    pages = x["cache"].k.shape[0]
    before = torch.rand(pages, Hkv, page, generator=torch.Generator().manual_seed(2)).cuda() * 3
    args = (x["table"], x["starts"], x["totals"])
    got = lib.key_weights(x["q"], lse, x["cache"], *args, before.clone(), causal=causal, decay=decay)
    torch.cuda.synchronize()
    k, _ = values(x["cache"])
    want = ref.key_weights(f64(x["q"]), f64(lse), k, *map(host, args), host(before), causal, decay)
    check_weights(got, want, before)
    again = lib.key_weights(x["q"], lse, x["cache"], *args, before.clone(), causal=causal, decay=decay,
                            max_tokens=max(new), max_length=max(a + b for a, b in zip(new, ctx)))
    torch.cuda.synchronize()
    check_weights(again, want, before)
    # each row's probabilities add up to one
    gained = f64(got).sum() - np.where(want[2] > 0, 0, f64(got)).sum()
    kept = want[0].sum() - np.where(want[2] > 0, 0, want[0]).sum()
    assert abs(gained - kept) <= 1e-4 * kept


def test_key_weights_leave_the_rest_alone(lib):
    """Requests without queries, pages that are not there, keys past max_length, rows that see nothing."""
    x = attention_inputs(lib, [2, 0, 3], [70, 40, 90], 4, 2, 64, 16, BF)
    x["table"][0, 1] = -1
    x["table"][2, 0] = 10 ** 6
    _, lse = attend(lib, x)
    lse[2, 1] = -float("inf")
    weights = torch.rand(x["cache"].k.shape[0], 2, 16, device="cuda")
    got = lib.key_weights(x["q"], lse, x["cache"], x["table"], x["starts"], x["totals"], weights.clone(), max_length=80)
    torch.cuda.synchronize()
    k, _ = values(x["cache"])
    totals = host(x["totals"])
    want = ref.key_weights(f64(x["q"]), f64(lse), k, host(x["table"]), host(x["starts"]), totals, host(weights))
    exact, row = want[0], host(x["table"])[2]
    for j in range(80, totals[2]):
        exact[row[j // 16], :, j % 16] = host(weights)[row[j // 16], :, j % 16]
    check_weights(got, want, weights)
    few = lib.key_weights(x["q"], lse, x["cache"], x["table"], x["starts"], x["totals"], weights.clone(), max_tokens=1)
    torch.cuda.synchronize()
    assert torch.equal(few, weights)


# ---- eviction -------------------------------------------------------------------------------------------

def evict_inputs(lib, lengths, heads, d, page, spare=None, layout="phd", seed=0):
    g = torch.Generator().manual_seed(seed)
    ends = [-(-t // page) + (spare[n] if spare else n % 3) for n, t in enumerate(lengths)]
    pages = sum(ends) + 5
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(ends) + 2), -7, dtype=torch.int32)
    at = 0
    for n, e in enumerate(ends):
        table[n, :e] = order[at:at + e]
        at += e
    head = int(torch.randint(0, 5 * pages, (1,), generator=g))
    queue = torch.full((pages,), -9, dtype=torch.int32)
    for i in range(5):
        queue[(head + i) % pages] = order[at + i]
    weights = torch.rand(pages, heads, page, generator=g) ** 4
    weights[torch.rand(pages, heads, page, generator=g) < 0.2] = 0.25  # ties
    return dict(cache=make_cache(lib, pages, page, heads, d, layout, g), weights=weights.cuda(), table=table.cuda(),
                totals=i32(lengths), pages=i32([[e, 0] for e in ends]), queue=queue.cuda(),
                cursor=torch.tensor([head, head + 5, 3], device="cuda"))


def check_evict(lib, x, budget, limit, sinks, recent, **kw):
    before = [np.ascontiguousarray(host(t)) for t in x["cache"]]
    want = ref.evict(before, host(x["weights"]).copy(), host(x["table"]), host(x["totals"]), host(x["pages"]),
                     host(x["queue"]), host(x["cursor"]), budget, limit, sinks, recent)
    table = x["table"].clone()
    e = lib.evict(x["cache"], x["weights"], x["table"], x["totals"], x["pages"], x["queue"], x["cursor"],
                  budget=budget, limit=limit, sinks=sinks, recent=recent, **kw)
    torch.cuda.synchronize()
    got = (*x["cache"], x["weights"], x["queue"], e.totals, e.pages, e.cursor, e.evicted)
    names = (*x["cache"]._fields, "weights", "queue", "totals", "pages", "cursor", "evicted")
    for name, a, b in zip(names, got, (*want[0], *want[1:])):
        assert host(a).tobytes() == np.ascontiguousarray(b).tobytes(), name
    assert torch.equal(table, x["table"])
    return e


EVICT_CASES = [
    # lengths, heads, d, page, budget, limit, sinks, recent, layout
    ([100], 2, 64, 16, 40, 40, 4, 8, "phd"),
    ([40, 41, 39, 0, 200], 2, 128, 16, 40, 40, 0, 0, "phd"),
    ([500, 90, 300], 3, 96, 24, 77, 100, 5, 13, "kv"),
    ([700], 1, 256, 8, 1, 1, 0, 0, "phd"),
    ([700], 1, 32, 8, 64, 64, 32, 32, "wide"),       # nothing is chosen by weight
    ([333, 90], 2, 160, 1, 50, 60, 0, 50, "hpd"),
    ([65, 64, 63], 8, 64, 16, 64, 64, 0, 1, "phd"),  # one token goes
    ([1500] * 70, 1, 64, 32, 1400, 1499, 4, 100, "phd"),
    ([3000], 2, 128, 16, 2999, 2999, 1, 1, "hpd"),
    ([40000, 33000], 1, 32, 64, 20000, 20000, 3, 500, "phd"),  # more than a workgroup keeps
    ([40000, 20000], 1, 32, 5, 9000, 9000, 3, 50, "phd"),
    ([16000, 15001, 3000], 2, 64, 16, 2000, 2000, 4, 30, "hpd"),
    ([1500, 300, 260] * 24, 4, 128, 16, 200, 250, 4, 20, "phd"),  # many requests and heads
    ([901] * 70, 2, 96, 24, 77, 100, 5, 13, "kv"),
    ([1300, 900] * 33, 2, 256, 16, 600, 700, 1, 1, "wide"),
    ([700] * 130, 1, 64, 32, 699, 699, 0, 0, "hpd"),
]


@pytest.mark.parametrize("lengths,heads,d,page,budget,limit,sinks,recent,layout", EVICT_CASES)
def test_evict(lib, lengths, heads, d, page, budget, limit, sinks, recent, layout):
    print("evict", lengths[:4], heads, d, page, budget, limit, flush=True)
    x = evict_inputs(lib, lengths, heads, d, page, layout=layout)
    check_evict(lib, x, budget, limit, sinks, recent)


def test_evict_ties_and_odd_weights(lib):
    """Equal weights throughout, zeros of both signs, infinities, NaN, subnormals, negative ones."""
    odd = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), float("nan"), 1e-42, -1e-42, 3.0, -3.0, 3.0000002])
    for kind in range(3):
        x = evict_inputs(lib, [300, 200], 2, 64, 16, seed=kind)
        if kind == 0:
            x["weights"].fill_(1.5)
        elif kind == 1:
            x["weights"].zero_()
        else:
            pick = torch.randint(0, 10, x["weights"].shape, generator=torch.Generator().manual_seed(4))
            x["weights"].copy_(odd[pick])
        check_evict(lib, x, 70, 70, 3, 9)


def test_evict_pages_that_are_not_there(lib):
    """Tokens on them go first and move nowhere; nothing is written outside the cache."""
    x = evict_inputs(lib, [160, 100], 2, 64, 16)
    x["table"][0, 3], x["table"][0, 7] = -1, 10 ** 7
    check_evict(lib, x, 90, 90, 2, 5)


def test_evict_twice_and_with_given_outputs(lib):
    x = evict_inputs(lib, [300, 50], 2, 64, 16)
    N = 2
    out = lib.Eviction(i32([9] * N), i32([[9, 9]] * N), torch.zeros(3, dtype=torch.int64, device="cuda"), i32([9] * N))
    space = lib.evict_workspace(x["cache"], x["table"], budget=100)
    space.fill_(255)
    e = check_evict(lib, x, 100, 200, 4, 16, out=out, workspace=space, max_length=300)
    assert e is out and e.totals.tolist() == [100, 50] and e.evicted.tolist() == [200, 0]
    x.update(totals=e.totals, pages=e.pages, cursor=e.cursor)
    again = check_evict(lib, x, 100, 200, 4, 16)
    assert again.totals.tolist() == [100, 50] and again.evicted.tolist() == [0, 0]


# ---- long contexts of many requests: a workgroup's waves share a token's key heads -----------------------------

def widened(x, N, keys):
    """The same requests among N, the others without tokens, in a table with room for `keys` tokens of each."""
    page = x["cache"].k.shape[1]
    n, m = x["table"].shape
    table = torch.full((N, -(-keys // page)), -1, dtype=torch.int32, device="cuda")
    table[:n, :m] = x["table"]
    last = x["starts"][-1:]
    return dict(x, table=table, starts=torch.cat((x["starts"], last.expand(N - n))).contiguous(),
                totals=torch.cat((x["totals"], torch.zeros(N - n, dtype=torch.int32, device="cuda"))))


LONG_CASES = [
    # new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype, N, keys
    ([1, 1, 1, 1], [0, 31, 700, 2000], 16, 4, 64, 16, 0, 0, True, BF, 64, 8192),
    ([1, 1, 1], [33, 1500, 800], 32, 8, 128, 16, 0, 0, True, HF, 64, 8192),
    ([2, 1], [1000, 63], 8, 4, 256, 32, 0, 0, True, BF, 64, 8192),
    ([4, 3], [900, 40], 32, 4, 128, 48, 0, 0, False, BF, 64, 8208),
    ([4, 2, 0, 1], [500, 1200, 9, 0], 32, 4, 64, 16, 0, 0, True, HF, 64, 8192),
    ([16, 9], [700, 90], 16, 4, 128, 16, 0, 0, True, BF, 64, 8192),
    ([16, 5], [300, 1100], 8, 2, 64, 16, 0, 0, False, HF, 128, 8192),
    ([8, 2], [400, 900], 8, 2, 256, 16, 0, 0, True, BF, 128, 8192),
    ([1, 1, 1], [300, 90, 33], 16, 4, 128, 16, 64, 4, True, BF, 8192, 400),
    ([4, 4], [300, 70], 32, 4, 64, 16, 40, 3, True, HF, 8192, 400),
    ([16, 16], [200, 333], 16, 4, 128, 32, 90, 20, True, BF, 8192, 400),
    ([2], [200], 32, 4, 256, 16, 33, 0, True, HF, 8192, 400),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,window,sinks,causal,dtype,N,keys", LONG_CASES)
def test_many_keys_in_all(lib, new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype, N, keys):
    print("many keys", new[:4], ctx[:4], Hq, Hkv, d, page, window, sinks, flush=True)
    x = attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype)
    mask = dict(window=window, sinks=sinks, causal=causal)
    y = widened(x, N, keys)
    got = attend(lib, y, **mask, max_tokens=max(new), max_length=keys)
    check_attention(x, got, wanted(x, **mask))
    if window:
        return
    before = torch.rand(x["cache"].k.shape[0], Hkv, page, generator=torch.Generator().manual_seed(2)).cuda()
    weights = lib.key_weights(y["q"], got[1], y["cache"], y["table"], y["starts"], y["totals"], before.clone(),
                              causal=causal, decay=0.75, max_tokens=max(new), max_length=keys)
    torch.cuda.synchronize()
    want = ref.key_weights(f64(x["q"]), f64(got[1]), values(x["cache"])[0],
                           *(host(x[k]) for k in ("table", "starts", "totals")), host(before), causal, 0.75)
    check_weights(weights, want, before)


@pytest.mark.parametrize("d,tokens", [(64, 1), (128, 4), (128, 16), (256, 8)])
def test_many_keys_with_gaps_and_nan(lib, d, tokens):
    """Pages that are not there, NaN blocks behind the end and at a place that the last query alone sees."""
    x = attention_inputs(lib, [tokens], [600], 16, 4, d, 16, BF)
    x["table"][0, 2], x["table"][0, 20], x["table"][0, 21] = -1, 10 ** 6, -5
    want = wanted(x)
    clean = attend(lib, widened(x, 64, 8192), max_tokens=tokens)
    check_attention(x, clean, want)
    c, row, total = x["cache"], host(x["table"])[0], 600 + tokens
    own = (row[(total - 1) // 16], (total - 1) % 16)
    c.v_scales[own[0], own[1], 1, 0] = 255
    for j in range(total, -(-total // 16) * 16):
        c.v_scales[row[j // 16], j % 16] = 255
        c.k_scales[row[j // 16], j % 16] = 255
    out, lse = attend(lib, widened(x, 64, 8192), max_tokens=tokens)
    nan = torch.zeros_like(out, dtype=torch.bool)
    nan[tokens - 1, 4:8, :32] = True
    assert torch.equal(out.isnan(), nan) and torch.equal(out[~nan], clean[0][~nan]) and torch.equal(lse, clean[1])


# ---- offsets past 32 bits, streams, graphs -----------------------------------------------------------------------

def far_cache(lib, x, pages):
    """The same cache at the other end of a large one: page p is page pages - 1 - p. -> x with it"""
    c = x["cache"]
    big = [torch.empty(pages, *t.shape[1:], dtype=torch.uint8, device="cuda") for t in c]
    for t, b in zip(c, big):
        b[pages - t.shape[0]:] = t.flip(0)
    return dict(x, cache=lib.Cache4(*big), table=torch.where(x["table"] < 0, -1, pages - 1 - x["table"]).to(torch.int32))


def test_offsets_past_32_bits(lib):
    """Pages 5 GB into a cache, and queries as far apart: bit for bit what the same ones near the front give."""
    pages = 600_000
    for new, ctx, N, keys in (([5, 1, 16], [300, 90, 0], 3, 400), ([1, 2], [300, 700], 64, 8192), ([70], [40], 1, 200)):
        print("far", new, flush=True)
        near = widened(attention_inputs(lib, new, ctx, 32, 8, 128, 16, BF), N, keys)
        far = far_cache(lib, near, pages)
        T = near["q"].shape[0]
        room = torch.empty(T, 1 << 26, dtype=BF, device="cuda")[:, :32 * 128].unflatten(1, (32, 128))
        room.copy_(near["q"])
        far["q"] = room
        got = [attend(lib, x, max_tokens=max(new)) for x in (near, far)]
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        w = [torch.zeros(x["cache"].k.shape[0], 8, 16, device="cuda") for x in (near, far)]
        for x, y in zip((near, far), w):
            lib.key_weights(x["q"], got[0][1], x["cache"], x["table"], x["starts"], x["totals"], y, max_tokens=max(new))
        torch.cuda.synchronize()
        n = w[0].shape[0]
        assert torch.equal(w[0], w[1][pages - n:].flip(0)) and not w[1][:pages - n].any()
        del room, far, w
    x = evict_inputs(lib, [500, 90], 8, 128, 16)
    far = far_cache(lib, x, pages)
    n = x["weights"].shape[0]
    far["weights"] = torch.zeros(pages, 8, 16, device="cuda")
    far["weights"][pages - n:] = x["weights"].flip(0)
    far["queue"] = x["queue"].clone()
    args = ("weights", "table", "totals", "pages", "queue", "cursor")
    for y in (x, far):
        lib.evict(y["cache"], *(y[k] for k in args), budget=77, sinks=3, recent=9)
    q, k, v, slots, positions, cs, _, w = rope_inputs(lib, 40, 16, 8, 128, 128, BF)
    slots = torch.arange(40, dtype=torch.int32, device="cuda") + 32
    lib.qk_norm_rope4(q, k, v, slots, positions, cs, x["cache"], q_weight=w[0], k_weight=w[1])
    there = (pages - 1 - slots // 16) * 16 + slots % 16
    lib.qk_norm_rope4(q, k, v, there.to(torch.int32), positions, cs, far["cache"], q_weight=w[0], k_weight=w[1])
    torch.cuda.synchronize()
    for a, b in zip((*x["cache"], x["weights"]), (*far["cache"], far["weights"])):
        assert torch.equal(a, b[pages - n:].flip(0))


def step_inputs(lib, seed):
    """One decoding step of three requests: what all four calls need, and where their results go."""
    x = evict_inputs(lib, [300, 500, 70], 4, 128, 16, seed=seed)
    new = [4, 1, 2]
    T, starts = sum(new), [0, 4, 5, 7]
    q, k, v, _, _, cs, _, w = rope_inputs(lib, T, 16, 4, 128, 128, BF, seed=seed)
    total, table = host(x["totals"]), host(x["table"])
    at = [(n, total[n] - new[n] + i) for n in range(3) for i in range(new[n])]
    x.update(q=q, k=k, v=v, cs=cs, w=w, starts=i32(starts), slots=i32([table[n, j // 16] * 16 + j % 16 for n, j in at]),
             positions=i32([j for _, j in at]), turned=torch.zeros(T, 16, 128, dtype=BF, device="cuda"),
             out=torch.zeros(T, 16, 128, dtype=BF, device="cuda"), lse=torch.zeros(T, 16, device="cuda"),
             made=lib.Eviction(i32([0] * 3), i32([[0, 0]] * 3), torch.zeros(3, dtype=torch.int64, device="cuda"), i32([0] * 3)))
    x["ws"] = lib.window_attention4_workspace(x["turned"], x["cache"], x["table"], max_tokens=4)
    x["ews"] = lib.evict_workspace(x["cache"], x["table"], budget=100)
    x["start"] = [t.clone() for t in (*x["cache"], x["weights"], x["queue"])]
    return x


def reset(x):
    for t, s in zip((*x["cache"], x["weights"], x["queue"]), x["start"]):
        t.copy_(s)
    for t in (x["turned"], x["out"], x["lse"], *x["made"]):
        t.zero_()


def run_step(lib, x):
    lib.qk_norm_rope4(x["q"], x["k"], x["v"], x["slots"], x["positions"], x["cs"], x["cache"], q_weight=x["w"][0],
                      k_weight=x["w"][1], out=x["turned"])
    lib.window_attention4(x["turned"], x["cache"], x["table"], x["starts"], x["totals"], max_tokens=4, lse=x["lse"],
                          out=x["out"], workspace=x["ws"])
    lib.key_weights(x["turned"], x["lse"], x["cache"], x["table"], x["starts"], x["totals"], x["weights"], decay=0.9,
                    max_tokens=4)
    lib.evict(x["cache"], x["weights"], x["table"], x["totals"], x["pages"], x["queue"], x["cursor"], budget=100,
              sinks=4, recent=16, out=x["made"], workspace=x["ews"])


def results(x):
    return [t.clone() for t in (*x["cache"], x["weights"], x["queue"], x["turned"], x["out"], x["lse"], *x["made"])]


def test_steps_on_two_streams(lib):
    steps = [step_inputs(lib, s) for s in (1, 2)]
    want = []
    for x in steps:
        run_step(lib, x)
        torch.cuda.synchronize()
        want.append(results(x))
    streams = [torch.cuda.Stream() for _ in steps]
    for again in range(3):
        for x, s in zip(steps, streams):
            with torch.cuda.stream(s):
                reset(x)
                run_step(lib, x)
        torch.cuda.synchronize()
        for x, w in zip(steps, want):
            assert all(map(torch.equal, results(x), w))


def test_captured_steps(lib):
    """Two graphs that share their workspaces, replayed in turn, with eager steps between."""
    steps = [step_inputs(lib, s) for s in (3, 4)]
    steps[1]["ws"], steps[1]["ews"] = steps[0]["ws"], steps[0]["ews"]
    want, graphs = [], []
    for x in steps:
        run_step(lib, x)
        torch.cuda.synchronize()
        want.append(results(x))
    for x in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run_step(lib, x)
        graphs.append(g)
    for again in range(3):
        for x in steps:
            reset(x)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, w in zip(steps, want):
            assert all(map(torch.equal, results(x), w)), again
        reset(steps[again % 2])
        run_step(lib, steps[again % 2])
        torch.cuda.synchronize()
        assert all(map(torch.equal, results(steps[again % 2]), want[again % 2]))
