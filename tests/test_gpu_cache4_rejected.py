"""GPU test: drafted tokens that are rejected leave nothing in the keys' weights. A layer of examples/long_context_serving.py
weighs its blocks when it is known how many tokens stay; the definition's weights are those of the accepted rows alone.
Tolerances as in test_gpu_cache4.py."""
import numpy as np
import pytest
import torch

import oracle.cache4 as ref
from test_gpu_cache4 import check_weights, f64, host, values
from test_gpu_cache4_example import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_rejected_tokens_weigh_nothing(lib, example):  # noqa: F811
    N, hidden = 3, 64
    layer = example.BudgetLayer(N, hidden, 4, 2, 64, pages=40, page_size=8, longest=96, positions=400, budget=80, limit=96,
                                sinks=3, recent=10, decay=0.9, seed=2)
    g = torch.Generator(device="cuda").manual_seed(8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = lambda n: torch.randn(n, hidden, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    layer.step(x(73), i32([40, 3, 30]), 73, 40)
    for accepted in ([16, 1, 7], [5, 16, 2]):
        print("accepted", accepted, flush=True)
        before = layer.weights.clone()
        layer.step(x(48), i32([16] * N), 48, 16, weigh=False)
        assert torch.equal(layer.weights, before)
        layer.weigh(i32(accepted))
        torch.cuda.synchronize()
        q, lse, plan = layer.open[:3]
        kept = f64(lse)
        for n, a in enumerate(accepted):
            kept[16 * n + a:16 * (n + 1)] = -np.inf
        want = ref.key_weights(f64(q), kept, values(layer.cache)[0], host(layer.table), host(plan.starts), host(plan.totals),
                               host(before), True, 0.9)
        check_weights(layer.weights, want, before)
        layer.keep(layer.lengths - (16 - i32(accepted)))
