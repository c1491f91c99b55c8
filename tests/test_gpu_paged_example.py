"""GPU test: the serving loop of examples/paged_serving.py. Its calls together against one dense
computation: a layer is driven through prompts, blocks, rejections and ended requests, and every
step's output must be what attention over the tokens each request has kept gives, computed from their
hidden states with no cache, in 64 bits. Tolerance: the layer's bf16 roundings (projection, queries,
keys, probabilities, attention output, final product), each 2^-8 relative to values of size about one
after norms; a sum of such independent errors over the products stays below 0.06 of the output's
root mean square per element times six; the mean below a tenth of that."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle.paged as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _dense(layer, states, new):
    """states: a request's kept hidden states [n, hidden] with the `new` last ones being queries."""
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    x, w, table = f(states), f(layer.w_qkv), f(layer.cos_sin)
    n, d = x.shape[0], layer.d
    y = (x @ w).reshape(n, layer.heads + 2 * layer.kv, d)
    cos, sin = table[:n, :d // 2], table[:n, d // 2:]
    q = ref.norm_rope(y[:, :layer.heads], f(layer.q_weight), cos, sin, 1e-6, False)
    k = ref.norm_rope(y[:, layer.heads:layer.heads + layer.kv], f(layer.k_weight), cos, sin, 1e-6, False)
    v = y[:, layer.heads + layer.kv:]
    first = n - new
    return ref.attention(q[first:], k[None], v[None], np.zeros((1, 1), np.int64), [0, new], [n],
                         layer.window, layer.sinks)[0].reshape(new, -1) @ f(layer.w_out)


@pytest.mark.parametrize("shared,window", [(0, 24), (0, 0), (40, 0)])
def test_steps_match_a_dense_layer(lib, example, shared, window):
    N, hidden, P = 3, 64, 8
    layer = example.PagedLayer(N, hidden, 4, 2, 64, pages=60, page_size=P, longest=160, window=window,
                               sinks=3 if window else 0, shared=shared, seed=1)
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda n: torch.randn(n, hidden, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    prompt = r(shared)
    if shared:
        layer.write_shared(prompt)
    kept = [prompt for _ in range(N)]
    for step, (new, accepted) in enumerate([((50, 3, 0), None), ((7, 7, 7), (7, 2, 5)), ((1, 1, 1), None),
                                            ((0, 9, 40), (0, 9, 11)), ((6, -1, 6), None), ((5, 12, 5), None)]):
        print("step", step, new, flush=True)
        counts = [max(n, 0) for n in new]
        x = r(sum(counts))
        before = layer.lengths
        y = layer.step(x, torch.tensor(new, dtype=torch.int32, device="cuda"), sum(counts), max(counts))
        torch.cuda.synchronize()
        parts = x.split(counts)
        for n, out in enumerate(y.split(counts)):
            if new[n] < 0:
                kept[n] = prompt
                continue
            kept[n] = torch.cat((kept[n], parts[n]))
            if not counts[n]:
                continue
            want = _dense(layer, kept[n], counts[n])
            err = np.abs(out.double().cpu().numpy() - want)
            rms = np.sqrt(np.mean(want ** 2))
            assert err.max() < 0.36 * rms and err.mean() < 0.036 * rms, (step, n, err.max() / rms, err.mean() / rms)
        if accepted:
            layer.keep(before + torch.tensor(accepted, dtype=torch.int32, device="cuda"))
            kept = [k[:len(k) - c + a] for k, c, a in zip(kept, counts, accepted)]
    assert int(layer.cursor[2]) == 0


def test_serving_loop_runs_and_repeats(lib, example):
    for shared in (0, 100):
        a, layer = example.serve(steps=4, N=4, V=5000, prompt=60, shared=shared)
        b, _ = example.serve(steps=4, N=4, V=5000, prompt=60, shared=shared)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and int(a.min()) >= 0 and int(a.max()) < 5000
        assert int(layer.cursor[2]) == 0
