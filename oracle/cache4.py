"""Plain definitions of the 4-bit paged cache's calls (lilicorr_qk_norm_rope4, lilicorr_window_attention4,
lilicorr_key_weights, lilicorr_evict): loops over requests, heads and tokens, numpy doubles. Test infrastructure
only; shares no code with the HIP path."""
from __future__ import annotations

import numpy as np

from . import paged

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(x):
    """x [.., d] doubles -> codes [.., d / 2] and scales [.., d / 32], uint8."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    codes, scales = np.zeros(blocks.shape, np.uint8), np.zeros(len(blocks), np.uint8)
    for i, b in enumerate(blocks):
        if not np.isfinite(b).all():
            scales[i] = 255
            continue
        e = -126
        while e < 125 and np.abs(b).max() > 7 * 2.0 ** e:
            e += 1
        far = np.abs(np.abs(b)[:, None] / 2.0 ** e - VALUES)
        for k in range(32):
            near = np.nonzero(far[k] == far[k].min())[0]
            even = [c for c in near if c % 2 == 0]
            codes[i, k] = (even[0] if len(near) > 1 else near[0]) + (8 if np.signbit(b[k]) else 0)
        scales[i] = e + 127
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | codes[..., 1::2] << 4, scales.reshape(*x.shape[:-1], x.shape[-1] // 32)


def values(codes, scales):
    """What codes [.., d / 2] and scales [.., d / 32] stand for, doubles [.., d]. 255 is NaN; 0, 253 and 254, which have no
    meaning, are 2^-127 and NaN here."""
    n = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    s = np.where(scales >= 253, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return np.where(n > 7, -1, 1) * VALUES[n & 7] * np.repeat(s, 32, -1)


def seen(j, p, total, causal, window=0, sinks=0):
    return 0 <= j < total and (not causal or j <= p) and (not window or j > p - window or j < sinks)


def attention(q, k, v, table, starts, totals, **mask):
    """k, v as `values` gives them. -> paged.attention's four results and lse [T, heads] (-inf where nothing is
    seen). NaN in keys or values reaches the rows that see them, and of those only the elements concerned."""
    out, absolute, sizes, count = paged.attention(q, k, v, table, starts, totals, **mask)
    T, heads, d = q.shape
    pages, P, kv, _ = k.shape
    lse = np.full((T, heads), -np.inf)
    for n in range(len(totals)):
        new = int(starts[n + 1]) - int(starts[n])
        for i in range(new):
            t, p = int(starts[n]) + i, int(totals[n]) - new + i
            js = [j for j in range(min(int(totals[n]), table.shape[1] * P))
                  if seen(j, p, int(totals[n]), mask.get("causal", True), mask.get("window", 0), mask.get("sinks", 0))
                  and 0 <= table[n, j // P] < pages]
            for h in range(heads):
                s = [k[table[n, j // P], j % P, h // (heads // kv)] @ q[t, h] / np.sqrt(d) for j in js]
                if s:
                    lse[t, h] = max(s) + np.log(np.sum(np.exp(np.array(s) - max(s))))
    return out, absolute, sizes, count, lse


def key_weights(q, lse, k, table, starts, totals, weights, causal=True, decay=1.0, scale=None):
    """-> the new weights [pages, kv, P], and of each the sum of its terms times an estimate of their magnitude
    (1 + |score| + sum |q k| + |lse|) for error bounds, and how many terms it has."""
    T, heads, d = q.shape
    pages, P, kv, _ = k.shape
    scale = 1 / np.sqrt(d) if scale is None else scale
    out, size = weights.astype(np.float64).copy(), np.zeros(weights.shape)
    terms = np.zeros(weights.shape, np.int64)
    for n in range(len(totals)):
        new, total = int(starts[n + 1]) - int(starts[n]), int(totals[n])
        if not new:
            continue
        for j in range(min(total, table.shape[1] * P)):
            page, o = int(table[n, j // P]), j % P
            if not 0 <= page < pages:
                continue
            for h in range(kv):
                w = decay * float(weights[page, h, o]) if j < total - new else 0.0
                for i in range(new):
                    if causal and j > total - new + i:
                        continue
                    for g in range(h * (heads // kv), (h + 1) * (heads // kv)):
                        t = int(starts[n]) + i
                        if lse[t, g] == -np.inf:
                            continue
                        s = scale * (q[t, g] @ k[page, o, h])
                        e = np.exp(s - lse[t, g])
                        w += e
                        size[page, h, o] += e * (1 + scale * (np.abs(q[t, g]) @ np.abs(k[page, o, h])) + abs(lse[t, g]))
                        terms[page, h, o] += 1
                out[page, h, o] = w
    return out, size, terms


def evict(parts, weights, table, totals, pages, queue, cursor, budget, limit, sinks, recent):
    """parts: arrays [pages, P, kv, ..] that move with the tokens. -> (parts, weights, queue, totals, pages, cursor,
    evicted), none of them the inputs."""
    n_pages, kv, P = weights.shape
    parts, old, old_w = [x.copy() for x in parts], parts, weights
    weights, queue = weights.copy(), queue.copy()
    totals_out, pages_out, evicted, tail = [], [], [], int(cursor[1])
    for n in range(len(totals)):
        end = min(max(int(pages[n][0]), 0), table.shape[1])
        L = max(min(int(totals[n]), end * P), 0)
        if L <= limit:
            totals_out.append(L)
            pages_out.append((end, int(pages[n][1])))
            evicted.append(0)
            continue
        place = [(int(table[n, j // P]), j % P) for j in range(L)]
        for h in range(kv):
            def rank(j):
                page, o = place[j]
                if not 0 <= page < n_pages:
                    return (0, 0.0)
                w = old_w[page, h, o]
                if np.isnan(w):
                    return (0, 0.0) if np.signbit(w) else (2, 0.0)
                return (1, float(w))
            middle = sorted(range(sinks, L - recent), key=rank, reverse=True)  # stable: earlier ones first
            kept = sorted([*range(sinks), *middle[:budget - sinks - recent], *range(L - recent, L)])
            assert len(kept) == budget
            for i, j in enumerate(kept):
                if not (0 <= place[j][0] < n_pages and 0 <= place[i][0] < n_pages):
                    continue
                for new, x in zip(parts, old):
                    new[place[i]][h] = x[place[j]][h]
                weights[place[i][0], h, place[i][1]] = old_w[place[j][0], h, place[j][1]]
        left = -(-budget // P)
        for e in range(left, end):
            queue[tail % len(queue)] = table[n, e]
            tail += 1
        totals_out.append(budget)
        pages_out.append((left, int(pages[n][1])))
        evicted.append(L - budget)
    i32 = np.int32
    return (parts, weights, queue, np.array(totals_out, i32), np.array(pages_out, i32),
            np.array([cursor[0], tail, cursor[2]], np.int64), np.array(evicted, i32))
