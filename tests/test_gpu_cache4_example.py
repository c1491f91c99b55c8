"""GPU test: the serving loop of examples/long_context_serving.py. Its calls together against one dense computation:
a layer is driven through prompts, blocks, rejections, evictions and ended requests, and every step's output must be
what attention over the keys and values that each head has kept gives. The dense side keeps for every request and
head the list of its tokens as 64-bit numbers: keys and values computed from the hidden states, rounded to 4 bits by
the definition; it adds the weights up itself and follows the library's choice of tokens (which near ties may turn
either way), checking that what the library let go is not heavier than what it kept.

Tolerances: the projection's bf16 rounding and sums may change a code by one step, so the dense side takes the
projection's output as the layer made it. What is left are the roundings of queries, probabilities and the attention's
output to bf16, each 2^-8 relative, against values of size about one: scores move by at most 2^-8 sum |q k| / sqrt(d), about
2^-8 * 5, and with them the output by 0.04 of its size at most; the output product adds up such independent errors.
Bounds as in the unquantised loop's test: 0.06 of the output's root mean square per element times six, the mean below
a tenth of that. Weights: a score's error of 0.02 is 2 percent of a weight, over a run of steps the same; 6 percent and
1e-3 are asked for."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle.cache4 as ref
import oracle.paged

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("long_context_serving",
                                                  os.path.join(ROOT, "examples", "long_context_serving.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class Dense:
    """One request: per key head the kept tokens' keys, values, weights, and what position is next."""

    def __init__(self, layer):
        self.layer, self.next = layer, 0
        self.heads = [dict(k=np.zeros((0, layer.d)), v=np.zeros((0, layer.d)), w=np.zeros(0)) for _ in range(layer.kv)]

    def step(self, y):
        """y [new, heads + 2 kv, d]: the projection's output -> the attention's output [new, heads * d]"""
        a, new = self.layer, len(y)
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        at = self.next + np.arange(new)
        cos, sin = f(a.cos_sin)[at, :a.d // 2], f(a.cos_sin)[at, a.d // 2:]
        self.next += new
        q = oracle.paged.norm_rope(y[:, :a.heads], f(a.q_weight), cos, sin, 1e-6, False)
        k = oracle.paged.norm_rope(y[:, a.heads:a.heads + a.kv], f(a.k_weight), cos, sin, 1e-6, False)
        k, v = (ref.values(*ref.quantise(t)) for t in (k, y[:, a.heads + a.kv:]))
        out = np.zeros((new, a.heads, a.d))
        for h, kept in enumerate(self.heads):
            before = len(kept["w"])
            kept["k"], kept["v"] = np.concatenate((kept["k"], k[:, h])), np.concatenate((kept["v"], v[:, h]))
            kept["w"] = np.concatenate((kept["w"] * a.decay, np.zeros(new)))
            for i in range(new):
                for g in range(h * (a.heads // a.kv), (h + 1) * (a.heads // a.kv)):
                    s = kept["k"][:before + i + 1] @ q[i, g] / np.sqrt(a.d)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[i, g] = p @ kept["v"][:before + i + 1]
                    kept["w"][:before + i + 1] += p
        return out.reshape(new, -1)

    def drop(self, count):
        """Its last `count` tokens are rejected."""
        self.next -= count
        for kept in self.heads:
            for name in kept:
                kept[name] = kept[name][:len(kept[name]) - count]


def stored(layer, n):
    """Of request n and each key head: keys, values, weights as the cache holds them."""
    row, P = layer.table[n].cpu().numpy(), layer.page_size
    at = [(row[j // P], j % P) for j in range(int(layer.lengths[n]))]
    c = [t.cpu().numpy() for t in layer.cache]
    k, v = ref.values(c[0], c[1]), ref.values(c[2], c[3])
    w = layer.weights.double().cpu().numpy()
    rows = lambda t, h: np.array([t[p, o, h] for p, o in at]).reshape(-1, layer.d)  # noqa: E731
    return [dict(k=rows(k, h), v=rows(v, h), w=np.array([w[p, h, o] for p, o in at])) for h in range(layer.kv)]


def check_stored(layer, n, want):
    for got, kept in zip(stored(layer, n), want.heads):
        assert got["w"].shape == kept["w"].shape
        assert np.array_equal(got["k"], kept["k"]) and np.array_equal(got["v"], kept["v"])
        assert (np.abs(got["w"] - kept["w"]) <= 0.06 * kept["w"] + 1e-3).all()


def follow_eviction(layer, n, want):
    """The dense side keeps what the library kept, after checking it: a subsequence, the first and last ones in it, none that
    went heavier than one that was chosen."""
    b = layer.bounds
    for got, kept in zip(stored(layer, n), want.heads):
        size = len(kept["w"])
        if size <= b["limit"]:
            assert len(got["w"]) == size
            continue
        assert len(got["w"]) == b["budget"]
        chosen, j = [], 0
        for i in range(b["budget"]):
            while not (np.array_equal(kept["k"][j], got["k"][i]) and np.array_equal(kept["v"][j], got["v"][i])):
                j += 1  # (past the end: not a subsequence)
            chosen.append(j)
            j += 1
        assert chosen[:b["sinks"]] == list(range(b["sinks"]))
        assert chosen[len(chosen) - b["recent"]:] == list(range(size - b["recent"], size))
        middle = [i for i in chosen if b["sinks"] <= i < size - b["recent"]]
        gone = [i for i in range(b["sinks"], size - b["recent"]) if i not in chosen]
        assert max(kept["w"][gone]) <= min(kept["w"][middle]) * 1.13 + 2e-3  # 6 percent either way
        for name in kept:
            kept[name] = kept[name][chosen]


def test_steps_match_a_dense_layer(lib, example):
    N, hidden = 3, 64
    layer = example.BudgetLayer(N, hidden, 4, 2, 64, pages=60, page_size=8, longest=160, positions=400, budget=40, limit=56,
                                sinks=3, recent=10, decay=0.9, seed=1)
    g = torch.Generator(device="cuda").manual_seed(7)
    kept = [Dense(layer) for _ in range(N)]
    lost = 0
    for step, (new, accepted) in enumerate([((90, 3, 0), None), ((7, 7, 7), (7, 2, 5)), ((1, 1, 1), None),
                                            ((0, 9, 70), (0, 9, 60)), ((20, -1, 6), None), ((5, 12, 5), None),
                                            ((30, 60, 1), None), ((1, 1, 1), None)]):
        print("step", step, new, flush=True)
        counts = [max(n, 0) for n in new]
        x = torch.randn(sum(counts), hidden, generator=g, device="cuda").to(torch.bfloat16)
        projected = (x @ layer.w_qkv).double().cpu().numpy().reshape(len(x), -1, 64)
        y = layer.step(x, torch.tensor(new, dtype=torch.int32, device="cuda"), sum(counts), max(counts)).double().cpu().numpy()
        at = 0
        for n in range(N):
            if new[n] < 0:
                kept[n] = Dense(layer)
            if counts[n]:
                want = kept[n].step(projected[at:at + counts[n]]) @ layer.w_out.double().cpu().numpy()
                err, rms = np.abs(y[at:at + counts[n]] - want), np.sqrt(np.mean(want ** 2))
                assert err.max() < 0.36 * rms and err.mean() < 0.036 * rms, (step, n, err.max() / rms, err.mean() / rms)
            at += counts[n]
            check_stored(layer, n, kept[n])
        if accepted:
            layer.keep(layer.lengths - torch.tensor([c - a for c, a in zip(counts, accepted)], device="cuda"))
            for d, c, a in zip(kept, counts, accepted):
                d.drop(c - a)
        before = layer.gone.clone()
        layer.cut()
        lost += int((layer.gone - before).sum())
        for n in range(N):
            follow_eviction(layer, n, kept[n])
            check_stored(layer, n, kept[n])
            assert int(layer.lengths[n] + layer.gone[n]) == kept[n].next
    assert lost > 100 and int(layer.cursor[2]) == 0
    held = sum(-(-int(t) // 8) for t in layer.lengths)
    assert int(layer.cursor[1] - layer.cursor[0]) == 60 - held  # every other page is free


def test_serving_loop_runs_and_repeats(lib, example):
    a, layer = example.serve(steps=6, N=4, V=5000, prompt=200)
    b, _ = example.serve(steps=6, N=4, V=5000, prompt=200)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and int(a.min()) >= 0 and int(a.max()) < 5000
    assert int(layer.cursor[2]) == 0 and int(layer.lengths.max()) <= 192 and int(layer.gone.max()) > 0
