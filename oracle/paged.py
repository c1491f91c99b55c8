"""Plain definitions of the paged-cache calls (lilicorr_page_plan, lilicorr_qk_norm_rope,
lilicorr_window_attention, lilicorr_prefix_attention): loops over requests, tokens and heads,
Python integers and numpy doubles. Test infrastructure only; shares no code with the HIP path."""
from __future__ import annotations

import numpy as np


def page_plan(lengths, incoming, pages, table, queue, cursor, page_size, tokens, window=0, sinks=0):
    """One request after the other, one page after the other. table and queue are not changed; the
    new ones come back with the other outputs. Tokens for which there was no page are not part of their
    request: it holds at most as many as its pages do. Nor are the ones past the `tokens`-th row."""
    P, M, C = page_size, table.shape[1], len(queue)
    table, queue = table.copy(), queue.copy()
    head, tail = int(cursor[0]), int(cursor[1])
    first = -(-sinks // P) if window else 0
    free = [int(queue[i % C]) for i in range(head, tail)]
    taken = lacking = 0
    back, pages_out, starts, totals, slots, positions = [], [], [0], [], [], []
    for n, (L, new) in enumerate(zip(map(int, lengths), map(int, incoming))):
        end, since = int(pages[n][0]), max(int(pages[n][1]), first)
        if new < 0:
            back += [int(table[n, e]) for e in range(end) if e < first or e >= since]
            pages_out.append((0, 0))
            totals.append(0)
            starts.append(starts[-1])
            continue
        L = min(L, end * P)
        # entries whose every token is behind the first query's window
        gone = []
        if window:
            gone = [e for e in range(since, end) if (e + 1) * P - 1 <= L - window]
        back += [int(table[n, e]) for e in gone]
        held = end
        for e in range(end, min(-(-(L + new) // P), M)):
            if taken < len(free):
                table[n, e] = free[taken]
                taken += 1
                held += 1
            else:
                table[n, e] = -1
                lacking += 1
        rows = min(new, tokens - starts[-1])
        for p in range(L, L + rows):
            e = p // P
            page = int(table[n, e]) if e < held else -1
            slots.append(page * P + p % P if page >= 0 else -1)
            positions.append(p)
        pages_out.append((held, since + len(gone)))
        totals.append(L + rows)
        starts.append(starts[-1] + rows)
    for i, page in enumerate(back):
        queue[(tail + i) % C] = page
    pad = [-1] * (tokens - len(slots))
    i32 = np.int32
    return {"table": table, "queue": queue, "pages": np.array(pages_out, i32),
            "cursor": np.array([head + taken, tail + len(back), lacking], np.int64),
            "starts": np.array(starts, i32), "totals": np.array(totals, i32),
            "slots": np.array(slots + pad, i32), "positions": np.array(positions + pad, i32)}


def norm_rope(x, weight, angles_cos, angles_sin, eps, interleaved):
    """x [T, heads, d] -> normed and rotated, [T, heads, d] doubles; cos, sin [T, rot / 2]."""
    y = np.array(x, np.float64)
    half = angles_cos.shape[1]
    for t in range(y.shape[0]):
        for h in range(y.shape[1]):
            r = y[t, h]
            if weight is not None:
                r = r / np.sqrt(np.mean(r * r) + eps) * weight
            out = r.copy()
            for i in range(half):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
                c, s = angles_cos[t, i], angles_sin[t, i]
                out[a] = r[a] * c - r[b] * s
                out[b] = r[a] * s + r[b] * c
            y[t, h] = out
    return y


def attention(q, k_cache, v_cache, table, starts, totals, window=0, sinks=0, causal=True, scale=None,
              shared_table=None, shared_length=0):
    """-> (out [T, heads, d], sum_j p_j |v_j| of the same shape, largest sum |q_i k_i| of a row's
    visible keys [T, heads], visible keys [T]); the last three are for error bounds. Rows outside
    starts are zero."""
    T, heads, d = q.shape
    pages, P, kv, _ = k_cache.shape
    group = heads // kv
    scale = 1 / np.sqrt(d) if scale is None else scale
    out, absolute = np.zeros((T, heads, d)), np.zeros((T, heads, d))
    sizes, count = np.zeros((T, heads)), np.zeros(T, np.int64)
    for n in range(len(totals)):
        new = int(starts[n + 1]) - int(starts[n])
        for i in range(new):
            t = int(starts[n]) + i
            p = int(totals[n]) - new + i
            places = []
            for j in range(shared_length):
                places.append((int(shared_table[j // P]), j % P))
            for j in range(int(totals[n])):
                if causal and j > p:
                    continue
                if window and j <= p - window and j >= sinks:
                    continue
                if j // P >= table.shape[1]:
                    continue
                places.append((int(table[n, j // P]), j % P))
            places = [x for x in places if 0 <= x[0] < pages]
            count[t] = len(places)
            if not places:
                continue
            pg, of = np.array(places).T
            k, v = k_cache[pg, of], v_cache[pg, of]  # [keys, kv, d]
            for h in range(heads):
                s = k[:, h // group] @ q[t, h] * scale
                sizes[t, h] = np.max(np.abs(k[:, h // group]) @ np.abs(q[t, h])) * scale
                e = np.exp(s - s.max())
                e /= e.sum()
                out[t, h] = e @ v[:, h // group]
                absolute[t, h] = e @ np.abs(v[:, h // group])
    return out, absolute, sizes, count
