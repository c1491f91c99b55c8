"""GPU tests of the paged-cache calls against the plain 64-bit definitions (oracle/paged.py).

Tolerances, from the roundings that the calls make (u = 2^-8 for bf16, 2^-11 for fp16: half a unit in
the last place of significands of 8 and 11 bits, relative to the value):
  whole numbers and copies  equal
  norm_rope   u |y| for the one rounding, 1e-6 (|a| + |b|) <= 4e-6 max |row| for fp32 arithmetic
  attention   u |o| for the output, u sum p|v| for the probabilities, and for the fp32 scores an
              error e of at most 2^-24 ((d + 2) S + 4 |s|) with S = scale sum |q_i k_i| >= |s|, which
              moves the result by at most 2 e sum p|v|; the fp32 sums over n keys n 2^-23 sum p|v|
plus half the smallest fp16 number where that is the type.
"""
import numpy as np
import pytest
import torch

import oracle.paged as ref

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- page plan -------------------------------------------------------------------------------------

PLAN_CASES = {
    # name: (lengths, incoming, filled beyond ceil(L / P) or since, page, window, sinks, free pages, extra)
    "one token, empty cache": dict(lengths=[0], incoming=[1], page=16, free=3),
    "nothing comes": dict(lengths=[33, 0], incoming=[0, 0], page=16, free=3),
    "block ends on a page": dict(lengths=[16], incoming=[16], page=16, free=1),
    "page of one": dict(lengths=[3, 5], incoming=[4, 2], page=1, free=10),
    "odd page, prefill": dict(lengths=[0, 100, 7], incoming=[1000, 16, 16], page=24, free=60),
    "queue runs out": dict(lengths=[10, 20, 30], incoming=[40, 40, 40], page=8, free=6),
    "queue empty": dict(lengths=[8, 8], incoming=[1, 0], page=8, free=0),
    "table too narrow": dict(lengths=[30, 3], incoming=[40, 3], page=8, free=20, width=6),
    "window gives back": dict(lengths=[500, 90, 64, 65], incoming=[16, 16, 16, 16], page=16, free=9,
                              window=64, sinks=4),
    "window, no sinks": dict(lengths=[500, 63, 64], incoming=[1, 1, 1], page=16, free=9, window=48),
    "window, many sinks": dict(lengths=[500, 20], incoming=[8, 8], page=8, free=9, window=16, sinks=100),
    "ended": dict(lengths=[100, 50, 7], incoming=[-1, 16, -5], page=16, free=4),
    "ended behind a window": dict(lengths=[300, 300, 5], incoming=[-1, 2, -1], page=16, free=2, window=40,
                                  sinks=20, since={0: 12, 1: 12}),
    "rejected tokens kept their pages": dict(lengths=[17, 33], incoming=[16, 16], page=16, free=4,
                                             filled={0: 3, 1: 5}),
}


def _plan_inputs(c, seed=0):
    rng = np.random.default_rng(seed)
    P, N = c["page"], len(c["lengths"])
    window, sinks = c.get("window", 0), c.get("sinks", 0)
    pages = []
    for n, L in enumerate(c["lengths"]):
        pages.append((c.get("filled", {}).get(n, -(-L // P)), c.get("since", {}).get(n, 0)))
    width = c.get("width", max(-(-(L + max(i, 0)) // P) for L, i in zip(c["lengths"], c["incoming"])) + 2)
    pages = [(min(e, width), s) for e, s in pages]
    total = sum(e for e, _ in pages) + c["free"] + 3
    order = rng.permutation(total).astype(np.int32)
    table = np.full((N, width), -7, np.int32)
    at = 0
    for n, (e, _) in enumerate(pages):
        table[n, :e] = order[at:at + e]
        at += e
    head = int(rng.integers(0, 10 * total))
    queue = np.full(total, -9, np.int32)
    for i in range(c["free"]):
        queue[(head + i) % total] = order[at + i]
    tokens = sum(max(i, 0) for i in c["incoming"]) + c.get("extra", 5)
    return dict(lengths=np.array(c["lengths"], np.int32), incoming=np.array(c["incoming"], np.int32),
                pages=np.array(pages, np.int32), table=table, queue=queue,
                cursor=np.array([head, head + c["free"], 77], np.int64), page_size=P, tokens=tokens,
                window=window, sinks=sinks)


def _run_plan(lib, x):
    dev = {k: torch.from_numpy(v).cuda() for k, v in x.items() if isinstance(v, np.ndarray)}
    p = lib.page_plan(**dev, page_size=x["page_size"], tokens=x["tokens"], window=x["window"],
                      sinks=x["sinks"])
    torch.cuda.synchronize()
    got = {k: getattr(p, k).cpu().numpy() for k in p._fields}
    return dict(got, table=dev["table"].cpu().numpy(), queue=dev["queue"].cpu().numpy())


def _same(got, want):
    assert got.keys() == want.keys()
    for k in want:
        assert np.array_equal(got[k], want[k]), f"{k}:\n{got[k]}\n{want[k]}"


@pytest.mark.parametrize("name", PLAN_CASES)
def test_page_plan(lib, name):
    x = _plan_inputs(PLAN_CASES[name])
    _same(_run_plan(lib, x), ref.page_plan(**x))


@pytest.mark.parametrize("N,seed", [(1, 1), (63, 2), (64, 3), (257, 4), (1025, 5), (4096, 6)])
def test_page_plan_many_requests(lib, N, seed):
    rng = np.random.default_rng(seed)
    c = dict(lengths=rng.integers(0, 700, N).tolist(),
             incoming=np.where(rng.random(N) < 0.1, -1, rng.integers(0, 20, N)).tolist(), page=16,
             free=int(N * 0.8), window=200, sinks=5)
    x = _plan_inputs(c, seed)
    _same(_run_plan(lib, x), ref.page_plan(**x))


def test_page_plan_over_a_run(lib):
    """Twenty steps of a small server, each from what the last one left: every page is always either
    in one live place of one table or in the queue, and the outputs are the definition's."""
    rng = np.random.default_rng(9)
    P, N, W, S = 4, 6, 24, 3
    x = _plan_inputs(dict(lengths=[0] * N, incoming=[0] * N, page=P, free=80, width=40), 9)
    x.update(window=W, sinks=S)
    x["pages"][:] = 0
    total, lengths = len(x["queue"]), np.zeros(N, np.int64)
    alive = set(range(total)) & set(int(x["queue"][i % total]) for i in range(*map(int, x["cursor"][:2])))
    for step in range(20):
        new = rng.integers(0, 9, N)
        new[rng.random(N) < 0.1] = -1
        new[lengths + np.maximum(new, 0) > 150] = -1
        x.update(lengths=lengths.astype(np.int32), incoming=new.astype(np.int32),
                 tokens=int(np.maximum(new, 0).sum()))
        want, got = ref.page_plan(**x), _run_plan(lib, x)
        _same(got, want)
        assert want["cursor"][2] == 0
        # of the new tokens some are rejected
        lengths = np.where(new < 0, 0, lengths + rng.integers(0, np.maximum(new, 0) + 1))
        x.update({k: got[k] for k in ("pages", "table", "queue", "cursor")})
        held = []
        for n in range(N):
            end, since = got["pages"][n]
            held += [int(got["table"][n, e]) for e in range(end) if e < 1 or e >= since]
        free = [int(got["queue"][i % total]) for i in range(*map(int, got["cursor"][:2]))]
        assert sorted(held + free) == sorted(alive), step


# ---- norms and rotation ------------------------------------------------------------------------------

def _rope_inputs(T, Hq, Hkv, d, rot, dtype, norm=True, page=16, layout="phd", seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    qkv = r(T, (Hq + 2 * Hkv) * d).to(dtype).cuda()
    q, k, v = (qkv[:, a * d:b * d].view(T, b - a, d) for a, b in
               ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    pages = T // page * 2 + 3
    if layout == "phd":
        kc, vc = (r(pages, page, Hkv, d).to(dtype).cuda() for _ in range(2))
    elif layout == "hpd":  # heads outside the page's tokens
        kc, vc = (r(pages, Hkv, page, d).to(dtype).cuda().transpose(1, 2) for _ in range(2))
    else:  # keys and values of a page side by side
        kc, vc = r(pages, 2, page, Hkv, d).to(dtype).cuda().unbind(1)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    slots[T // 2:T // 2 + 1] = -1
    positions = torch.randint(0, 5000, (T,), generator=g).to(torch.int32)
    if T > 3:
        positions[3], slots[2] = -1, pages * page  # no token; a slot that is not there
        positions[1] = 5000                        # past the table
    ang = torch.rand(5000, max(rot // 2, 1), generator=g, dtype=torch.float64)[:, :rot // 2] * 6.3
    cs = torch.cat((ang.cos(), ang.sin()), 1).float().cuda() if rot else None
    w = [1 + 0.2 * r(d).cuda() if norm else None for _ in range(2)]
    return q, k, v, slots.cuda(), positions.cuda(), cs, kc, vc, w


ROPE_CASES = [
    # T, Hq, Hkv, d, rot, dtype, interleaved, norm, page, layout
    (1, 32, 8, 128, 128, torch.bfloat16, False, True, 16, "phd"),
    (1, 1, 1, 16, 16, torch.float16, True, True, 1, "phd"),
    (17, 8, 8, 64, 64, torch.bfloat16, False, True, 16, "hpd"),
    (33, 12, 4, 80, 80, torch.float16, False, True, 24, "kv"),
    (20, 6, 2, 96, 32, torch.bfloat16, False, True, 16, "phd"),
    (20, 5, 1, 256, 256, torch.bfloat16, False, False, 8, "phd"),
    (9, 14, 2, 248, 112, torch.float16, True, True, 16, "kv"),
    (7, 3, 3, 24, 16, torch.bfloat16, True, False, 16, "hpd"),
    (10, 4, 2, 128, 0, torch.float16, False, True, 16, "phd"),
    (600, 4, 1, 64, 64, torch.bfloat16, False, True, 16, "phd"),
    (4100, 2, 1, 32, 32, torch.bfloat16, False, True, 64, "phd"),
    # a token's heads spread over waves: each step, a third of them, two, none
    (150, 32, 8, 128, 128, torch.bfloat16, False, True, 16, "kv"),
    (301, 32, 8, 128, 64, torch.float16, True, True, 16, "phd"),
    (303, 5, 3, 200, 80, torch.bfloat16, False, True, 16, "phd"),
    (2101, 8, 2, 128, 128, torch.bfloat16, False, True, 16, "hpd"),
    (6150, 3, 1, 96, 96, torch.float16, False, True, 32, "phd"),
]


@pytest.mark.parametrize("T,Hq,Hkv,d,rot,dtype,inter,norm,page,layout", ROPE_CASES)
def test_qk_norm_rope(lib, T, Hq, Hkv, d, rot, dtype, inter, norm, page, layout):
    q, k, v, slots, positions, cs, kc, vc, w = _rope_inputs(T, Hq, Hkv, d, rot, dtype, norm, page, layout)
    before = f64(kc), f64(vc)
    out = lib.qk_norm_rope(q, k, v, slots, positions, cs, kc, vc, q_weight=w[0], k_weight=w[1],
                           eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    pos, sl = positions.cpu().numpy(), slots.cpu().numpy()
    live = (pos >= 0) & (pos < 5000) if rot else pos >= 0
    at = np.where(live, pos, 0)
    table = f64(cs) if rot else np.zeros((5001, 0))
    c, s = table[at, :rot // 2], table[at, rot // 2:]
    want = [ref.norm_rope(f64(x), f64(y) if y is not None else None, c, s, 1e-5, inter)
            for x, y in ((q, w[0]), (k, w[1]))]

    def close(got, exact, what):
        tol = U[dtype] * np.abs(exact) + 4e-6 * np.abs(exact).max(-1, keepdims=True) + TINY[dtype]
        bad = ~(np.abs(got - exact) <= tol)
        assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first {np.argwhere(bad)[0]}"

    want[0][~live] = 0
    close(f64(out), want[0], "q")
    kf, vf = before
    P = kc.shape[1]
    stored = live & (sl >= 0) & (sl < kc.shape[0] * P)
    gk, gv = f64(kc), f64(vc)
    for t in np.nonzero(stored)[0]:
        close(gk[sl[t] // P, sl[t] % P], want[1][t], f"k of token {t}")
        assert np.array_equal(gv[sl[t] // P, sl[t] % P], f64(v[t])), f"v of token {t}"
        gk[sl[t] // P, sl[t] % P], gv[sl[t] // P, sl[t] % P] = kf[sl[t] // P, sl[t] % P], vf[sl[t] // P, sl[t] % P]
    assert np.array_equal(gk, kf) and np.array_equal(gv, vf), "a slot that no token has was written"


def test_qk_norm_rope_in_place(lib):
    q, k, v, slots, positions, cs, kc, vc, w = _rope_inputs(40, 8, 2, 128, 128, torch.bfloat16, seed=3)
    q = q.contiguous()
    args = (slots, positions, cs, kc, vc)
    want = lib.qk_norm_rope(q, k, v, *args, q_weight=w[0], k_weight=w[1])
    got = lib.qk_norm_rope(q, k, v, *args, q_weight=w[0], k_weight=w[1], out=q)
    torch.cuda.synchronize()
    assert got is q and torch.equal(got, want)


def test_qk_norm_rope_no_tokens(lib):
    q, k, v, slots, positions, cs, kc, vc, w = _rope_inputs(4, 4, 2, 64, 64, torch.bfloat16)
    kept = kc.clone()
    out = lib.qk_norm_rope(q[:0], k[:0], v[:0], slots[:0], positions[:0], cs, kc, vc)
    torch.cuda.synchronize()
    assert out.shape == (0, 4, 64) and torch.equal(kc, kept)


# ---- attention -----------------------------------------------------------------------------------------

def _attention_inputs(new, ctx, Hq, Hkv, d, page, dtype, shared=0, layout="phd", seed=0, pad_rows=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    totals = [a + b for a, b in zip(new, ctx)]
    counts = [-(-t // page) for t in totals]
    sp = -(-shared // page)
    pages = sum(counts) + sp + 3
    order = torch.randperm(pages, generator=g)
    width = max(max(counts), 1) + 1
    table = torch.full((len(new), width), -1, dtype=torch.int32)
    at = sp
    for n, c in enumerate(counts):
        table[n, :c] = order[at:at + c]
        at += c
    starts = np.concatenate(([0], np.cumsum(new))).tolist()
    T = starts[-1] + pad_rows
    sharp = (0.5 * 2.0 ** (torch.arange(Hq) % 4))[None, :, None]
    q = (r(T, Hq, d) * sharp).to(dtype).cuda()
    if layout == "phd":
        kc, vc = (r(pages, page, Hkv, d).to(dtype).cuda() for _ in range(2))
    elif layout == "hpd":
        kc, vc = (r(pages, Hkv, page, d).to(dtype).cuda().transpose(1, 2) for _ in range(2))
    else:
        kc, vc = r(pages, 2, page, Hkv, d).to(dtype).cuda().unbind(1)
    return dict(q=q, k_cache=kc, v_cache=vc, table=table.cuda(), starts=i32(starts), totals=i32(totals),
                shared_table=order[:sp].to(torch.int32).cuda())


def _want(x, shared=0, **mask):
    return ref.attention(f64(x["q"]), f64(x["k_cache"]), f64(x["v_cache"]), x["table"].cpu().numpy(),
                         x["starts"].cpu().numpy(), x["totals"].cpu().numpy(),
                         shared_table=x["shared_table"].cpu().numpy(), shared_length=shared, **mask)


def _attend(lib, x, shared=0, **kw):
    a = (x["q"], x["k_cache"], x["v_cache"])
    b = (x["table"], x["starts"], x["totals"])
    if shared:
        return lib.prefix_attention(*a, x["shared_table"], shared, *b, **kw)
    return lib.window_attention(*a, *b, **kw)


def _check(x, got, want):
    exact, absolute, sizes, count = want
    dtype, d = x["q"].dtype, x["q"].shape[2]
    u = U[dtype]
    e = 2.0 ** -24 * ((d + 2) * sizes + 4 * sizes)
    tol = u * np.abs(exact) + (u + 2 * e + count[:, None] * 2.0 ** -23)[..., None] * absolute + TINY[dtype]
    bad = ~(np.abs(f64(got) - exact) <= tol)
    assert not bad.any(), (f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: "
                           f"{f64(got)[bad][0]!r} for {exact[bad][0]!r}, bound {tol[bad][0]!r}")


BF, HF = torch.bfloat16, torch.float16
WINDOW_CASES = [
    # new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype
    ([1], [0], 1, 1, 64, 16, 0, 0, True, BF),
    ([1], [700], 32, 8, 128, 16, 0, 0, True, BF),
    ([1], [700], 32, 8, 128, 16, 100, 4, True, BF),
    ([1, 1, 1], [0, 31, 32], 4, 2, 64, 8, 0, 0, True, HF),
    ([1, 1, 1, 1], [63, 64, 65, 300], 8, 8, 128, 1, 64, 1, True, BF),
    ([16, 16], [100, 333], 32, 8, 128, 16, 0, 0, True, BF),
    ([16, 16], [100, 333], 32, 8, 128, 16, 50, 7, True, HF),
    ([16], [400], 8, 2, 64, 16, 33, 64, False, BF),
    ([16, 3, 0, 1], [0, 5, 77, 260], 7, 1, 64, 24, 0, 0, False, HF),
    ([0, 33, 1, 17], [9, 200, 0, 64], 14, 2, 64, 24, 90, 7, False, HF),
    ([150], [0], 4, 1, 128, 16, 0, 0, True, BF),
    ([150, 70], [33, 500], 4, 1, 128, 32, 40, 3, True, BF),
    ([65], [70], 2, 2, 80, 24, 0, 0, True, HF),
    ([40, 5], [70, 300], 6, 2, 96, 128, 64, 16, True, BF),
    ([1, 2], [500, 40], 16, 2, 256, 16, 0, 0, True, BF),
    ([16, 7], [300, 90], 8, 2, 256, 16, 60, 4, True, HF),
    ([50], [90], 4, 1, 256, 16, 0, 0, True, BF),
    ([3], [20], 6, 2, 16, 4, 0, 0, True, HF),
    ([3, 20], [40, 60], 5, 1, 200, 16, 30, 2, True, BF),
    ([1], [2000], 16, 1, 64, 16, 1, 0, True, BF),     # a window of the query alone
    ([2, 9], [50, 50], 64, 1, 64, 16, 0, 0, True, BF),  # 64 query heads to a key head
    ([1] * 70, list(range(70)), 4, 2, 64, 16, 0, 0, True, BF),
    ([1, 90] * 35, list(range(70)), 2, 1, 64, 16, 33, 2, True, BF),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,window,sinks,causal,dtype", WINDOW_CASES)
def test_window_attention(lib, new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype):
    print("window attention", new[:4], ctx[:4], Hq, Hkv, d, page, window, sinks, flush=True)
    x = _attention_inputs(new, ctx, Hq, Hkv, d, page, dtype)
    mask = dict(window=window, sinks=sinks, causal=causal)
    got = _attend(lib, x, max_tokens=max(new), max_length=int(x["totals"].max()), **mask)
    want = _want(x, **mask)
    _check(x, got, want)
    # bounds that the host does not know: the same rows, other tiles and chunks
    _check(x, _attend(lib, x, **mask), want)


PREFIX_CASES = [
    # new, ctx, shared, Hq, Hkv, d, page, causal, dtype
    ([1], [0], 1, 1, 1, 64, 16, True, BF),
    ([1, 1, 1], [0, 40, 200], 300, 32, 8, 128, 16, True, BF),
    ([16, 16, 16], [1, 40, 20], 500, 8, 2, 128, 16, True, HF),
    ([5, 0, 9, 1], [0, 30, 7, 300], 77, 12, 4, 80, 24, True, HF),
    ([4, 3], [10, 0], 1000, 6, 2, 64, 16, False, BF),
    ([20, 7], [10, 0], 130, 4, 2, 256, 32, True, BF),
    ([1] * 40, [0] * 40, 65, 3, 1, 96, 8, True, BF),
]


@pytest.mark.parametrize("new,ctx,shared,Hq,Hkv,d,page,causal,dtype", PREFIX_CASES)
def test_prefix_attention(lib, new, ctx, shared, Hq, Hkv, d, page, causal, dtype):
    print("prefix attention", new[:4], ctx[:4], shared, Hq, Hkv, d, page, flush=True)
    x = _attention_inputs(new, ctx, Hq, Hkv, d, page, dtype, shared=shared)
    want = _want(x, shared, causal=causal)
    _check(x, _attend(lib, x, shared, causal=causal, max_tokens=max(new),
                      max_length=int(x["totals"].max())), want)
    _check(x, _attend(lib, x, shared, causal=causal), want)


@pytest.mark.parametrize("layout", ["hpd", "kv"])
def test_attention_strided(lib, layout):
    x = _attention_inputs([16, 1], [90, 200], 8, 2, 128, 16, BF, layout=layout)
    wide = torch.randn(17, 12, 128, dtype=BF, device="cuda")
    wide[:, 2:10] = x["q"]
    x["q"] = wide[:, 2:10]
    _check(x, _attend(lib, x, window=64, sinks=3), _want(x, window=64, sinks=3))


def test_attention_scale_and_repeat(lib):
    """A scale of one's own; the same bits on every call, workspace kept, and on a stream of its own."""
    x = _attention_inputs([3, 1], [900, 40], 8, 2, 64, 16, HF)
    ws = lib.window_attention_workspace(x["q"], x["k_cache"], x["table"])
    first = _attend(lib, x, scale=0.03, workspace=ws)
    _check(x, first, _want(x, scale=0.03))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(5):
            assert torch.equal(_attend(lib, x, scale=0.03, workspace=ws), first)


def test_attention_rows_that_see_nothing(lib):
    """Pages that are not there, totals below the queries, no keys at all: zeros, finite everywhere."""
    x = _attention_inputs([4, 4, 2], [60, 0, 30], 4, 2, 64, 16, BF, pad_rows=3)
    x["table"][0, 1:3] = -1
    x["table"][0, 3] = x["k_cache"].shape[0]  # past the cache
    x["table"][2, :] = -1
    x["totals"][1] = 2  # its first two queries lie before the first key
    for window, sinks in ((0, 0), (8, 2)):
        mask = dict(window=window, sinks=sinks)
        out = torch.full_like(x["q"], 5.0)
        got = _attend(lib, x, out=out, **mask)
        want = _want(x, **mask)
        assert (want[3][:10] == 0).sum() >= 4
        assert (f64(got)[10:] == 5).all(), "rows past the last request were written"
        trimmed = dict(x, q=x["q"][:10])
        _check(trimmed, got[:10], tuple(w[:10] for w in want))


@pytest.mark.parametrize("fill", [float("inf"), float("-inf"), float("nan"), 3e38])
@pytest.mark.parametrize("new,ctx", [([16], [100]), ([1, 1], [100, 40]), ([80], [20])])
def test_attention_unseen_values(lib, fill, new, ctx):
    """What a row does not see has no effect on it: unlisted pages, the rest of the last page, keys
    behind the window, and later tokens of the same block."""
    x = _attention_inputs(new, ctx, 4, 2, 128, 16, BF, seed=4)
    mask = dict(window=40, sinks=5)
    P, table = 16, x["table"].cpu().numpy()
    seen = torch.zeros(x["k_cache"].shape[:2], dtype=torch.bool)
    at = 0
    for n, (t, c) in enumerate(zip(new, ctx)):
        for j in range(t + c):
            if j > c - 40 or j < 5:
                seen[table[n, j // P], j % P] = True
    # the block's last token: its own row alone sees it
    own = [(int(table[n, (t + c - 1) // P]), (t + c - 1) % P) for n, (t, c) in enumerate(zip(new, ctx))]
    for name in ("k_cache", "v_cache"):
        x[name][~seen.cuda()] = fill
    clean = dict(x, k_cache=torch.nan_to_num(x["k_cache"], 0, 0, 0).clamp(-100, 100),
                 v_cache=torch.nan_to_num(x["v_cache"], 0, 0, 0).clamp(-100, 100))
    want = _want(clean, **mask)
    _check(x, _attend(lib, x, **mask), want)
    for pg, of in own:
        x["v_cache"][pg, of] = fill
        x["k_cache"][pg, of, :, 0] = fill
    got = _attend(lib, x, **mask)
    last = np.cumsum(new) - 1
    others = np.setdiff1d(np.arange(sum(new)), last)
    if len(others):
        _check(dict(x, q=x["q"][others]), got[others], tuple(w[others] for w in want))


def test_attention_nan_reaches_its_rows(lib):
    x = _attention_inputs([4], [30], 2, 1, 64, 16, BF)
    x["q"][1, 0] = float("nan")
    table = x["table"].cpu().numpy()
    x["v_cache"][int(table[0, 2]), 1, 0, 7] = float("nan")  # key 33, seen by the last query alone
    got = f64(_attend(lib, x))
    assert np.isnan(got[1, 0]).all()
    assert np.isnan(got[3, :, 7]).all() and np.isnan(got).sum() == 64 + 2


def test_attention_long_offsets(lib):
    """Cache offsets past 2^32 bytes: the pages of one request lie at both ends of a 9 GB cache."""
    P, pages = 16, 9 * (1 << 30) // (16 * 2 * 128 * 2)
    k = torch.zeros(pages, P, 2, 128, dtype=BF, device="cuda")
    x = _attention_inputs([16], [80], 4, 2, 128, P, BF)
    small = x["table"][0, :6].tolist()
    far = [pages - 1, 3, pages // 2, pages - 2, 0, pages - 7]
    v = k  # values are the keys themselves
    for a, b in zip(small, far):
        k[b] = x["k_cache"][a]
    x["v_cache"] = x["k_cache"]
    want = _want(x)
    y = dict(x, k_cache=k, v_cache=v, table=torch.full_like(x["table"], -1))
    y["table"][0, :6] = i32(far)
    _check(x, _attend(lib, y), want)


@pytest.mark.parametrize("less", [12.3, 16.6, 20.4, 21.6, 23.7])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_many_small_probabilities(lib, less, dtype):
    """One key whose score stands above 65535 equal ones by a factor of 2^less in the powers, with the same
    value as theirs or none: the small ones must count as much as their number makes them. Many requests
    with the same pages, so that the keys are split little. Relative errors: u for the output; u for the
    rounded probabilities, or 2^(less - 32) where a type with steps of 2^-24 holds powers of up to 2^7; 1e-4
    for the scores (at most 24, in powers of two) and sums."""
    N, n, d, page = 1024, 1 << 16, 64, 64
    k = torch.zeros(n // page, page, 1, d, dtype=dtype, device="cuda")
    v = torch.ones_like(k)
    q = torch.zeros(N, 1, d, dtype=dtype, device="cuda")
    q[:, 0, 3] = 1.0
    k[700, 41, 0, 3] = 1.0
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(N, 1)
    small = (n - 1) * 2.0 ** -less
    rel = U[dtype] + max(U[dtype], 2.0 ** (less - 32) if dtype is torch.float16 else 0.0) + 1e-4
    for value in (0.0, 1.0):
        v[700, 41] = value
        o = lib.window_attention(q, k, v, table, i32(range(N + 1)), i32([n] * N), max_tokens=1,
                                 scale=less * float(np.log(2.0)))
        want = (small + value) / (small + 1.0)
        assert (o.double() - want).abs().max().item() <= rel * want + TINY[dtype]


def test_calls_in_a_graph(lib):
    """Captured once and replayed with other inputs, with eager work between the replays: the same bits as
    the eager calls on the same inputs. The attentions split their keys, so the join is recorded too."""
    new, ctx, shared = [16, 1, 7, 16], [900, 700, 0, 333], 650
    x = _attention_inputs(new, ctx, 8, 2, 128, 16, torch.bfloat16, seed=5)
    y = _attention_inputs(new, ctx, 8, 2, 128, 16, torch.bfloat16, shared=shared, seed=6)
    q, k, v, slots, positions, cs, kc, vc, w = _rope_inputs(40, 8, 2, 128, 128, torch.bfloat16)
    moved = (x["q"], y["q"], q, k, v, slots)
    keep, totals = [t.clone() for t in moved], x["totals"].clone()

    def calls():
        a = lib.qk_norm_rope(q, k, v, slots, positions, cs, kc, vc, q_weight=w[0], k_weight=w[1])
        return a, kc.clone(), _attend(lib, x, window=300, sinks=3), _attend(lib, y, shared=shared)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for replay in range(4):
        for t, t0 in zip(moved, keep):
            t.copy_(t0.roll(replay, 0))
        x["totals"].copy_(totals - replay)
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in got]
        for a, b in zip(first, calls()):
            assert torch.equal(a, b), replay
